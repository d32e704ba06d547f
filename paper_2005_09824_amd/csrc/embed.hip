// Rows of a table for given tokens, and the gradient of the table: positions sorted by token, then for every
// row of the table the sum over its positions, in their order. See include/lfmmi.h for the formulas.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/lfmmi.h"
#include "layers.h"
#include "rows.h"
#include "vec16.h"

namespace lfmmi {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ int64_t token_at(const void* tokens, int bytes, uint32_t i)
{
    return bytes == 8 ? static_cast<const int64_t*>(tokens)[i] : static_cast<const int32_t*>(tokens)[i];
}

__device__ __forceinline__ bool inside(const SeqLengths& lens, uint32_t row, int T)
{
    return lens.n == 0 || (int)(row % (uint32_t)T) < lens.T[row / (uint32_t)T];
}

template <bool Wave>
__device__ __forceinline__ uint32_t of_wave(uint32_t v) { return Wave ? (uint32_t)__builtin_amdgcn_readfirstlane((int)v) : v; }
template <bool Wave>
__device__ __forceinline__ int64_t of_wave(int64_t v)
{
    return (int64_t)((uint64_t)of_wave<Wave>((uint32_t)((uint64_t)v >> 32)) << 32 | of_wave<Wave>((uint32_t)v));
}

// Workgroups take pieces of groups of rows: 2^lanes_log2 lanes a row, one chunk of eight values each, and `rows` rows that
// follow each other by the same lanes.
struct Tiles {
    int lanes_log2;
    uint32_t pieces;
    int64_t units;
};
Tiles tiles_of(int64_t groups, int D)
{
    const int chunks = (D + 7) / 8;
    Tiles t{0, 0, 0};
    while ((1 << t.lanes_log2) < kThreads && (1 << t.lanes_log2) < chunks) ++t.lanes_log2;
    const int at_once = kThreads >> t.lanes_log2;
    t.pieces = (uint32_t)((chunks + (1 << t.lanes_log2) - 1) >> t.lanes_log2);
    t.units = (groups + at_once - 1) / at_once * t.pieces;
    return t;
}
struct Place {
    int64_t group;
    int c;
};
template <bool Wave>
__device__ __forceinline__ Place place_of(const Tiles& t, int64_t unit)
{
    const int64_t g = t.pieces == 1 ? unit : unit / t.pieces;
    return {(g << (8 - t.lanes_log2)) + of_wave<Wave>(threadIdx.x >> t.lanes_log2),
            ((int)(unit - g * t.pieces) << t.lanes_log2) + ((int)threadIdx.x & ((1 << t.lanes_log2) - 1))};
}
static_assert(kThreads == 1 << 8, "place_of");
// Wave: a row has 64 lanes or more, so that what belongs to it is the same in all lanes of a wave, and is held and computed
// once: a division for every row's sequence, the products of its place.
template <typename F>
void by_wave(const Tiles& t, F&& f)
{
    if (t.lanes_log2 >= 6) f(std::true_type{});
    else f(std::false_type{});
}
int grid_of(int64_t units) { return (int)std::min<int64_t>(units, 1 << 20); }

// ---- forward

// Rows of 16 bits that a lane has on their way: a token, then its row, are two waits. Bound by HBM: 32,768 rows of 2,048 bf16 of a table of
// 65,536, a third of them padding, 32 us (134 MB written, 65 MB of the table read; 55 us with one row a lane, 39 with rows in vector registers).
constexpr int kEmbedRows = 4;

template <typename T, Width W, int Rows, bool Wave>
__global__ __launch_bounds__(kThreads) void k_embed(EmbedParams p, SeqLengths lens, Tiles tiles)
{
    using Store = typename T::Store;
    const uint32_t rows = (uint32_t)p.B * (uint32_t)p.T;
    const int chunks = (p.D + 7) / 8;
    for (int64_t u = blockIdx.x; u < tiles.units; u += gridDim.x) {
        const Place at = place_of<Wave>(tiles, u);
        if (at.c >= chunks) continue;
        const int64_t first = at.group * Rows;
        int64_t token[Rows];
        Raw<T> v[Rows];
#pragma unroll
        for (int k = 0; k < Rows; ++k)
            token[k] = first + k < rows && inside(lens, (uint32_t)(first + k), p.T)
                ? token_at(p.tokens, p.token_bytes, (uint32_t)(first + k)) : -1;
#pragma unroll
        for (int k = 0; k < Rows; ++k) token[k] = of_wave<Wave>(token[k]);
#pragma unroll
        for (int k = 0; k < Rows; ++k)
            if (token[k] >= 0 && token[k] < p.V)
                v[k] = raw_at<T, W>(static_cast<const Store*>(p.table) + token[k] * p.stride, at.c, p.D);
#pragma unroll
        for (int k = 0; k < Rows; ++k) {
            if (first + k >= rows) continue;
            const bool bad = token[k] >= p.V;
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = bad ? NAN : 0.f;
            if (token[k] >= 0 && !bad) {
                unpack_at<T, W>(v[k], at.c, p.D, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= p.scale;
            }
            store_at<T, W>(static_cast<Store*>(p.out) + (first + k) * p.D, at.c, p.D, f, p.once);
            if (p.status && at.c == 0) p.status[first + k] = bad ? 4 : 0;
        }
    }
}

// ---- sorting positions by token: digits of plan.bits bits, the lowest first, every pass keeps the order of equal
// digits. Keys are tokens; V where there is none, or none of the table. A workgroup takes a tile of positions, a wave a
// stretch of it, 64 at a time in order.

constexpr int kSort = 1024;
constexpr int kSortWaves = kSort / 64;

__device__ __forceinline__ uint32_t key_of(const EmbedGradParams& p, const SeqLengths& lens, uint32_t i, uint32_t from)
{
    const int64_t token = inside(lens, i, p.T) ? token_at(p.tokens, p.token_bytes, from + i) : -1;
    return token < 0 || token >= p.V ? (uint32_t)p.V : (uint32_t)token;
}

// Keys of some sequences of a call of many.
__global__ __launch_bounds__(kThreads) void k_embed_keys(EmbedGradParams p, SeqLengths lens, uint32_t from, uint32_t n,
                                                         uint32_t* keys)
{
    for (uint32_t i = blockIdx.x * kThreads + threadIdx.x; i < n; i += gridDim.x * kThreads)
        keys[from + i] = key_of(p, lens, i, from);
}

// Sums of the lanes up to each.
__device__ __forceinline__ uint32_t sums_upto(uint32_t v)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t w = __shfl_up(v, o, 64);
        if ((int)(threadIdx.x & 63) >= o) v += w;
    }
    return v;
}

// The places of a wave's 64 keys, in their order: `mine` says where the next of every digit goes, and is moved on. Lanes with
// equal digits find each other by a ballot on each bit.
__device__ __forceinline__ uint32_t take_place(uint32_t* mine, uint32_t digit, int bits, bool in)
{
    const int lane = threadIdx.x & 63;
    uint64_t same = __ballot(in);
    for (int b = 0; b < bits; ++b) {
        const bool bit = digit >> b & 1;
        const uint64_t set = __ballot(bit);
        same &= bit ? set : ~set;
    }
    volatile uint32_t* place = &mine[digit];
    uint32_t to = 0;
    if (in) to = *place + __popcll(same & ((1ull << lane) - 1));
    __builtin_amdgcn_wave_barrier();
    if (in && (same >> lane) == 1) *place = to + 1;  // the last of them
    __builtin_amdgcn_wave_barrier();
    return to;
}

// How many keys of a tile have a digit: hist[tile][digit]. Tokens: the keys are made here, of all sequences.
template <bool Tokens>
__global__ __launch_bounds__(kSort) void k_embed_count(EmbedGradParams p, SeqLengths lens, uint32_t* keys, uint32_t N,
                                                       int shift, uint32_t* hist)
{
    extern __shared__ uint32_t bins[];
    const int n = 1 << p.plan.bits;
    for (int i = threadIdx.x; i < n; i += kSort) bins[i] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * p.plan.tile, end = min((int64_t)N, first + p.plan.tile);
    for (int64_t i = first + threadIdx.x; i < end; i += kSort) {
        const uint32_t key = Tokens ? key_of(p, lens, (uint32_t)i, 0) : keys[i];
        if (Tokens) keys[i] = key;
        atomicAdd(&bins[key >> shift & (n - 1)], 1u);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kSort) hist[(int64_t)blockIdx.x * n + i] = bins[i];
}

// Keys of a tile to their places. Every workgroup adds up for itself how many keys have a smaller digit, or the same in an
// earlier tile. starts: of the only pass, whose digits are the tokens, or null.
__global__ __launch_bounds__(kSort) void k_embed_place(EmbedGradParams p, const uint32_t* keys, const uint32_t* order,
                                                       uint32_t N, int shift, const uint32_t* hist, uint32_t* keys_out,
                                                       uint32_t* order_out, uint32_t* starts)
{
    extern __shared__ uint32_t places[];  // [wave][digit]
    __shared__ uint32_t sums[kSortWaves];
    const int bits = p.plan.bits, n = 1 << bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t* mine = places + wave * n;
    const int64_t stretch = p.plan.tile / kSortWaves, first = (int64_t)blockIdx.x * p.plan.tile + wave * stretch;
    const int64_t end = min((int64_t)N, first + stretch);
    // (a tile's first strip stays in registers: of most calls it is the only one)
    const bool here = first + lane < end;
    const uint32_t key0 = here ? keys[first + lane] : 0, whence0 = here ? (order ? order[first + lane] : (uint32_t)(first + lane)) : 0;
    // a digit a thread: how many keys there are in all, and in the tiles before
    const int d = threadIdx.x;
    uint32_t all = 0, before = 0;
    if (d < n)
        for (int t = 0; t < p.plan.tiles; t += 16) {
            uint32_t h[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) h[k] = t + k < p.plan.tiles ? hist[(int64_t)(t + k) * n + d] : 0;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                all += h[k];
                if (t + k < (int)blockIdx.x) before += h[k];
            }
        }
    for (int i = threadIdx.x; i < n * kSortWaves; i += kSort) places[i] = 0;
    __syncthreads();
    if (here) atomicAdd(&mine[key0 >> shift & (n - 1)], 1u);
    for (int64_t i = first + 64 + lane; i < end; i += 64) atomicAdd(&mine[keys[i] >> shift & (n - 1)], 1u);
    const uint32_t upto = sums_upto(all);
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    if (d < n) {
        uint32_t at = upto - all + before;
        for (int w = 0; w < wave; ++w) at += sums[w];
        if (starts && d <= p.V && blockIdx.x == 0) starts[d] = at;  // (nothing lies before the first tile)
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t count = places[w * n + d];
            places[w * n + d] = at;
            at += count;
        }
    }
    __syncthreads();
    for (int64_t strip = first; strip < end; strip += 64) {
        const int64_t i = strip + lane;
        const bool in = i < end;
        uint32_t key = key0, whence = whence0;
        if (strip > first && in) {
            key = keys[i];
            whence = order ? order[i] : (uint32_t)i;
        }
        const uint32_t to = take_place(mine, key >> shift & (n - 1), bits, in);
        if (in) {
            keys_out[to] = key;
            order_out[to] = whence;
        }
    }
}

// All of it for at most kFew positions, by one workgroup in LDS; where the positions of every token begin too, of at most
// kFewTokens tokens. (A call, replayed: 2,000 positions of 512 fp32, a table of 2,000: 17 us, sorted by the kernels above 24,
// the beginnings by a kernel of their own 19. A table of 5,000: 20, 24 and 20; 2,048 positions of 256, a table of 30,000: 44, 30
// and 25.)
constexpr int kFew = 2 * kSort, kFewTokens = 2048;
__global__ __launch_bounds__(kSort) void k_embed_sort_few(EmbedGradParams p, SeqLengths lens, bool tokens, uint32_t N,
                                                          uint32_t* keys_out, uint32_t* order_out, uint32_t* starts)
{
    constexpr int kBits = 9, kStretch = kFew / kSortWaves;
    __shared__ uint32_t key[2][kFew], places[kSortWaves << kBits], sums[kSortWaves];
    __shared__ uint16_t order[2][kFew];
    const int bits = p.plan.bits, n = 1 << bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t* mine = places + wave * n;
    const uint32_t first = wave * kStretch, end = min(N, first + kStretch);
    for (uint32_t i = threadIdx.x; i < N; i += kSort) {
        key[0][i] = tokens ? key_of(p, lens, i, 0) : keys_out[i];
        order[0][i] = (uint16_t)i;
    }
    int now = 0;
    for (int pass = 0, shift = 0; pass < p.plan.passes; ++pass, shift += bits, now ^= 1) {
        for (int i = threadIdx.x; i < n * kSortWaves; i += kSort) places[i] = 0;
        __syncthreads();
        for (uint32_t i = first + lane; i < end; i += 64) atomicAdd(&mine[key[now][i] >> shift & (n - 1)], 1u);
        __syncthreads();
        const int d = threadIdx.x;
        uint32_t all = 0;
        if (d < n)
            for (int w = 0; w < kSortWaves; ++w) all += places[w * n + d];
        const uint32_t upto = sums_upto(all);
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        if (d < n) {
            uint32_t at = upto - all;
            for (int w = 0; w < wave; ++w) at += sums[w];
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t count = places[w * n + d];
                places[w * n + d] = at;
                at += count;
            }
        }
        __syncthreads();
        for (uint32_t strip = first; strip < end; strip += 64) {
            const bool in = strip + lane < end;
            const uint32_t k = in ? key[now][strip + lane] : 0;
            const uint32_t to = take_place(mine, k >> shift & (n - 1), bits, in);
            if (in) {
                key[now ^ 1][to] = k;
                order[now ^ 1][to] = order[now][strip + lane];
            }
        }
        __syncthreads();
    }
    for (uint32_t i = threadIdx.x; i < N; i += kSort) {
        keys_out[i] = key[now][i];
        order_out[i] = order[now][i];
    }
    if (p.V > kFewTokens) return;
    for (uint32_t v = threadIdx.x; v <= (uint32_t)p.V; v += kSort) {
        uint32_t lo = 0, hi = N;
        while (lo < hi) {
            const uint32_t mid = (lo + hi) / 2;
            if (key[now][mid] < v) lo = mid + 1;
            else hi = mid;
        }
        starts[v] = lo;
    }
}

// Where the positions of every token begin: by halves, first among one key in `step` that lie in LDS.
constexpr int kSamples = 1024;
__global__ __launch_bounds__(kThreads) void k_embed_starts(const uint32_t* keys, uint32_t N, int V, uint32_t* starts)
{
    __shared__ uint32_t samples[kSamples];
    const uint32_t step = (N + kSamples - 1) / kSamples, have = step ? (N + step - 1) / step : 0;
    for (uint32_t i = threadIdx.x; i < have; i += kThreads) samples[i] = keys[i * step];
    __syncthreads();
    for (int64_t v = (int64_t)blockIdx.x * kThreads + threadIdx.x; v <= V; v += (int64_t)gridDim.x * kThreads) {
        uint32_t lo = 0, hi = have;
        while (lo < hi) {
            const uint32_t mid = (lo + hi) / 2;
            if (samples[mid] < (uint32_t)v) lo = mid + 1;
            else hi = mid;
        }
        // the first sample that is not below v, and so behind the one before
        hi = (uint32_t)min((uint64_t)N, (uint64_t)lo * step);
        lo = lo > 0 ? (lo - 1) * step + 1 : 0;
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (keys[mid] < (uint32_t)v) lo = mid + 1;
            else hi = mid;
        }
        starts[v] = lo;
    }
}

// ---- sums of rows

template <typename T, Width W>
__device__ __forceinline__ Raw<T> row_of(const EmbedGradParams& p, uint32_t pos, int c)
{
    const uint32_t b = pos / (uint32_t)p.T;
    return raw_at<T, W>(static_cast<const typename T::Store*>(p.g) + (int64_t)b * p.stride_b +
                                (int64_t)(pos - b * (uint32_t)p.T) * p.stride_t, c, p.D);
}

// Adds the chunk of positions order[from..to - 1], in that order.
template <typename T, Width W, int AtOnce, bool Wave>
__device__ __forceinline__ void add_rows(const EmbedGradParams& p, const uint32_t* order, uint32_t from, uint32_t to,
                                         int c, float* s)
{
    for (uint32_t k = from; k < to; k += AtOnce) {
        Raw<T> v[AtOnce];
#pragma unroll
        for (int j = 0; j < AtOnce; ++j) v[j] = row_of<T, W>(p, of_wave<Wave>(order[min(k + j, to - 1)]), c);
#pragma unroll
        for (int j = 0; j < AtOnce; ++j) {
            if (k + j >= to) continue;
            float f[8];
            unpack_at<T, W>(v[j], c, p.D, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += f[i];
        }
    }
}

template <typename T, Width W>
__device__ __forceinline__ void write_grad(const EmbedGradParams& p, int64_t v, int c, const float* s)
{
    typename T::Store* out = static_cast<typename T::Store*>(p.grad) + v * p.D;
    float f[8];
    if (p.accumulate) load_at<T, W>(out, c, p.D, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = p.accumulate ? f[i] + s[i] * p.scale : s[i] * p.scale;
    store_at<T, W>(out, c, p.D, f, p.once);
}

// The sorted positions in pieces of kEmbedPiece: one that a token has as a whole is added up by itself. A token's row is the
// sum of its positions before its first such piece, its pieces, and the positions behind the last.
struct Segment {
    uint32_t from, to, first, last;  // positions; pieces first..last - 1 are the token's
};
__device__ __forceinline__ Segment segment_of(uint32_t from, uint32_t to)
{
    const uint32_t first = (uint32_t)(((uint64_t)from + kEmbedPiece - 1) / kEmbedPiece), last = to / kEmbedPiece;
    return {from, to, first, last};
}

// Such pieces, and the rows of the table that have none, those without a position among them. A lane has kGradRows rows of
// the table, and asks for the first position's row of each before it waits for one. Bound by HBM and by three waits in a row (a
// token's positions, a position, its row): 65,536 rows of 2,048 bf16 for 21,000 positions 78 us (268 MB written, 85 read), of which
// the writes alone take 42; eight rows a lane 5 us more, two 5 us more.
constexpr int kGradRows = 4;
template <typename T, Width W>
__global__ __launch_bounds__(kThreads) void k_embed_rows(EmbedGradParams p, Tiles rows, Tiles pieces, const uint32_t* starts,
                                                         const uint32_t* keys, const uint32_t* order, float* partials)
{
    const int chunks = (p.D + 7) / 8;
    const uint32_t whole = (uint32_t)p.plan.pieces;
    for (int64_t u = blockIdx.x; u < pieces.units + rows.units; u += gridDim.x) {
        if (u < pieces.units) {
            const Place at = place_of<false>(pieces, u);
            if (at.c >= chunks || at.group >= whole) continue;
            const uint32_t from = (uint32_t)at.group * kEmbedPiece, key = keys[from];
            if (key != keys[from + kEmbedPiece - 1] || key == (uint32_t)p.V) continue;
            float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            add_rows<T, W, 8, false>(p, order, from, from + kEmbedPiece, at.c, s);
            store_at<F32, W>(partials + at.group * p.D, at.c, p.D, s);
            continue;
        }
        const Place at = place_of<false>(rows, u - pieces.units);
        const int64_t v = at.group * kGradRows;
        if (at.c >= chunks || v >= p.V) continue;
        uint32_t begin[kGradRows + 1];
        Raw<T> first[kGradRows];
#pragma unroll
        for (int k = 0; k <= kGradRows; ++k) begin[k] = starts[min(v + k, (int64_t)p.V)];
#pragma unroll
        for (int k = 0; k < kGradRows; ++k) {
            const Segment g = segment_of(begin[k], begin[k + 1]);
            first[k] = no_values<T>();
            if (g.from < g.to && g.first >= g.last) first[k] = row_of<T, W>(p, order[g.from], at.c);
        }
#pragma unroll
        for (int k = 0; k < kGradRows; ++k) {
            const Segment g = segment_of(begin[k], begin[k + 1]);
            if (g.first < g.last || v + k >= p.V || (g.from == g.to && p.accumulate)) continue;
            float s[8];
            unpack_at<T, W>(first[k], at.c, p.D, s);
            if (g.from + 1 < g.to) add_rows<T, W, 4, false>(p, order, g.from + 1, g.to, at.c, s);
            write_grad<T, W>(p, v + k, at.c, s);
        }
    }
}

// Tokens with pieces: a workgroup has 64 chunks of a row, every wave a stretch of the pieces and of the positions before and
// behind them. It does so for the tokens whose first piece is one of kJoinPieces. (32,768 positions of 2,048 bf16: 11 us; 24 with a
// workgroup of eight waves for each piece, most of which are no token's first, and 15 for eight pieces.)
constexpr int kJoinWaves = 4, kJoinPieces = 2;
template <typename T, Width W>
__global__ __launch_bounds__(kJoinWaves * 64) void k_embed_join(EmbedGradParams p, int parts, int64_t units,
                                                                const uint32_t* starts, const uint32_t* keys,
                                                                const uint32_t* order, const float* partials)
{
    __shared__ float sums[kJoinWaves][64 * 8];
    constexpr int kEnds = kEmbedPiece / kJoinWaves;  // positions of a wave before the pieces, and behind
    const int lane = threadIdx.x & 63, wave = (int)of_wave<true>(threadIdx.x >> 6), chunks = (p.D + 7) / 8;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const uint32_t group = (uint32_t)(u / parts);
        const int c = (int)(u - (int64_t)group * parts) * 64 + lane;
        const uint32_t mine = group * kJoinPieces + lane;
        uint32_t v = (uint32_t)p.V;
        if (lane < kJoinPieces && mine < (uint32_t)p.plan.pieces) {
            const uint32_t at = mine * kEmbedPiece;
            v = keys[at];
            if (v != keys[at + kEmbedPiece - 1] || (mine > 0 && v == keys[at - kEmbedPiece])) v = (uint32_t)p.V;
        }
        for (uint64_t some = __ballot(v < (uint32_t)p.V); some; some &= some - 1) {
            const uint32_t token = (uint32_t)__builtin_amdgcn_readlane((int)v, __ffsll((unsigned long long)some) - 1);
            const Segment g = segment_of(of_wave<true>(starts[token]), of_wave<true>(starts[token + 1]));
            const uint32_t n = g.last - g.first, each = (n + kJoinWaves - 1) / kJoinWaves, to = min(n, (wave + 1) * each);
            const float* part = partials + (int64_t)g.first * p.D;
            float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (c < chunks) {
                const uint32_t head = g.from + wave * kEnds, tail = g.last * kEmbedPiece + wave * kEnds;
                add_rows<T, W, kEnds, true>(p, order, head, min(head + kEnds, g.first * kEmbedPiece), c, s);
                // A token of many positions has a long sum here: eight pieces are added up by themselves, and what is rounded away
                // where their sum is added is added up beside it. (Half a million positions of one value:
                // up to 110 millionths off with a plain sum, and 1,363 us for 640 columns against 1,051.)
                float lost[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                for (uint32_t i = wave * each; i < to; i += 8) {
                    Raw<F32> f[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        f[j] = raw_at<F32, W>(part + (int64_t)min(i + j, to - 1) * p.D, c, p.D);
                    float e[8][8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (i + j >= to) f[j] = no_values<F32>();
                        unpack_at<F32, W>(f[j], c, p.D, e[j]);
                    }
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        const float sum = ((e[0][x] + e[1][x]) + (e[2][x] + e[3][x])) + ((e[4][x] + e[5][x]) + (e[6][x] + e[7][x]));
                        const float upto = s[x] + sum, added = upto - s[x];
                        lost[x] += (s[x] - (upto - added)) + (sum - added);
                        s[x] = upto;
                    }
                }
#pragma unroll
                for (int x = 0; x < 8; ++x) s[x] += fabsf(lost[x]) < INFINITY ? lost[x] : 0.f;  // (s is no number either then)
                add_rows<T, W, kEnds, true>(p, order, tail, min(tail + kEnds, g.to), c, s);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sums[wave][e * 64 + lane] = s[e];
            __syncthreads();
            if (wave == 0 && c < chunks) {
                for (int w = 1; w < kJoinWaves; ++w)
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[e] += sums[w][e * 64 + lane];
                write_grad<T, W>(p, token, c, s);
            }
            __syncthreads();
        }
    }
}

template <typename U>
U* place(const EmbedGradParams& p, size_t at)
{
    return reinterpret_cast<U*>(static_cast<char*>(p.workspace) + at);
}

}  // namespace

hipError_t launch_embed(const EmbedParams& p, const SeqLengths& lens, int dtype, hipStream_t stream)
{
    const int64_t rows = (int64_t)p.B * p.T;
    // One row a lane, or four (us of bf16, replayed, its own rows in the caches / others each time): 1,000 of 1,024 2.5 / 3.3 one,
    // 3.3 / 4.0 four; 4,000 of 2,048 6.5 / 10.1 and 6.5 / 10.3; 8,000 of 1,024 6.5 / 9.8 and 6.5 / 9.6; 32,000 of 640 16.1 / 21.9 and
    // 13.8 / 17.8; 30,000 of 2,048 35 / 46 and 36 / 41. Rows of 32 bits have twice as much on its way: 1,000 of 1,024 3.1 / 4.1 and
    // 3.8 / 4.8; 32,000 of 640 24.6 / 32.4 and 25.3 / 32.4; 30,000 of 2,048 70 / 77 and 72 / 83.
    const bool few = dtype == LFMMI_F32 || rows * ((p.D + 2047) / 2048) < 4096;
    const Tiles t = tiles_of(few ? rows : (rows + kEmbedRows - 1) / kEmbedRows, p.D);
    by_type(dtype, [&](auto type) {
        by_width<true>(p.D, [&](auto whole) {
            using Type = decltype(type);
            constexpr Width kWidth = decltype(whole)::value;
            by_wave(t, [&](auto wave) {
                constexpr bool kWave = decltype(wave)::value;
                constexpr int kMany = Type::kVec == 8 ? kEmbedRows : 1;
                if (few) k_embed<Type, kWidth, 1, kWave><<<grid_of(t.units), kThreads, 0, stream>>>(p, lens, t);
                else k_embed<Type, kWidth, kMany, kWave><<<grid_of(t.units), kThreads, 0, stream>>>(p, lens, t);
            });
        });
    });
    return hipGetLastError();
}

EmbedPlan plan_embed(int64_t N, int V, int D)
{
    EmbedPlan p{};
    int bits = 1;  // of a key: V is one
    while (bits < 31 && (int64_t)V >> bits > 0) ++bits;
    p.passes = (bits + 8) / 9;  // (512 digits of 16 waves: 32 KB of LDS)
    p.bits = (bits + p.passes - 1) / p.passes;
    // tiles of 1,024 positions, or more, so that there are 128 at most: every workgroup looks at all tiles' counts
    const int64_t tile = std::max<int64_t>(kSort, (N + 127) / 128);
    p.tile = (int32_t)((tile + kSort - 1) / kSort * kSort);
    p.tiles = (int32_t)((N + p.tile - 1) / p.tile);
    p.pieces = (int32_t)(N / kEmbedPiece);
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t from = at;
        at += (bytes + 15) / 16 * 16;
        return from;
    };
    p.keys = take((size_t)N * 4 * 2);
    p.order = take((size_t)N * 4 * 2);
    p.hist = take(((size_t)p.tiles << p.bits) * 4);
    p.starts = take(((size_t)V + 1) * 4);
    p.partials = take((size_t)p.pieces * D * 4);
    p.bytes = at;
    return p;
}

hipError_t launch_embed_keys(const EmbedGradParams& p, const SeqLengths& lens, int b, int n, hipStream_t stream)
{
    const uint32_t count = (uint32_t)n * (uint32_t)p.T;
    const int grid = (int)std::min<int64_t>(((int64_t)count + kThreads - 1) / kThreads, 4096);
    k_embed_keys<<<grid, kThreads, 0, stream>>>(p, lens, (uint32_t)b * (uint32_t)p.T, count,
                                                place<uint32_t>(p, p.plan.keys));
    return hipGetLastError();
}

hipError_t launch_embed_grad(const EmbedGradParams& p, const SeqLengths* lens, int dtype, hipStream_t stream)
{
    const EmbedPlan& plan = p.plan;
    const uint32_t N = (uint32_t)p.B * (uint32_t)p.T;
    uint32_t* keys[2] = {place<uint32_t>(p, plan.keys), place<uint32_t>(p, plan.keys) + N};
    uint32_t* order[2] = {place<uint32_t>(p, plan.order), place<uint32_t>(p, plan.order) + N};
    uint32_t* hist = place<uint32_t>(p, plan.hist);
    uint32_t* starts = place<uint32_t>(p, plan.starts);
    float* partials = place<float>(p, plan.partials);
    int now = 0;
    const int bins = 4 << plan.bits;
    const bool few = N > 0 && N <= kFew;
    if (few)
        k_embed_sort_few<<<1, kSort, 0, stream>>>(p, lens ? *lens : SeqLengths{}, lens != nullptr, N, keys[0], order[0], starts);
    for (int pass = 0; !few && N > 0 && pass < plan.passes; ++pass, now ^= 1) {
        const int shift = pass * plan.bits;
        if (pass == 0 && lens)
            k_embed_count<true><<<plan.tiles, kSort, bins, stream>>>(p, *lens, keys[0], N, shift, hist);
        else
            k_embed_count<false><<<plan.tiles, kSort, bins, stream>>>(p, SeqLengths{}, keys[now], N, shift, hist);
        k_embed_place<<<plan.tiles, kSort, bins * kSortWaves, stream>>>(p, keys[now], pass ? order[now] : nullptr, N, shift,
                                                                        hist, keys[now ^ 1], order[now ^ 1],
                                                                        plan.passes == 1 ? starts : nullptr);
    }
    if (few ? p.V > kFewTokens : N == 0 || plan.passes > 1) {
        const int64_t v = ((int64_t)p.V + kThreads) / kThreads;
        k_embed_starts<<<(int)std::min<int64_t>(v, 2048), kThreads, 0, stream>>>(keys[now], N, p.V, starts);
    }
    const Tiles rows = tiles_of(((int64_t)p.V + kGradRows - 1) / kGradRows, p.D), pieces = tiles_of(plan.pieces, p.D);
    by_type(dtype, [&](auto type) {
        by_width<true>(p.D, [&](auto whole) {
            using T = decltype(type);
            constexpr Width kWidth = decltype(whole)::value;
            k_embed_rows<T, kWidth><<<grid_of(rows.units + pieces.units), kThreads, 0, stream>>>(
                p, rows, pieces, starts, keys[now], order[now], partials);
            if (plan.pieces == 0) return;
            const int parts = (p.D + 511) / 512;
            const int64_t units = ((int64_t)plan.pieces + kJoinPieces - 1) / kJoinPieces * parts;
            k_embed_join<T, kWidth><<<(int)std::min<int64_t>(units, 1 << 16), kJoinWaves * 64, 0, stream>>>(
                p, parts, units, starts, keys[now], order[now], partials);
        });
    });
    return hipGetLastError();
}

}  // namespace lfmmi
