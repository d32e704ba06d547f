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
constexpr int kWaves = kThreads / 64;

__device__ __forceinline__ int64_t token_at(const void* tokens, int bytes, uint32_t i)
{
    return bytes == 8 ? static_cast<const int64_t*>(tokens)[i] : static_cast<const int32_t*>(tokens)[i];
}

__device__ __forceinline__ bool inside(const SeqLengths& lens, uint32_t row, int T)
{
    return lens.n == 0 || (int)(row % (uint32_t)T) < lens.T[row / (uint32_t)T];
}

// Workgroups take pieces of rows: 2^lanes_log2 lanes a row, `chunks` of eight values each.
struct Tiles {
    int lanes_log2;
    uint32_t pieces;
    int64_t units;
};
template <int Chunks>
Tiles tiles_of(int64_t rows, int D)
{
    const int chunks = (D + 7) / 8;
    Tiles t{0, 0, 0};
    while ((1 << t.lanes_log2) < kThreads && (1 << t.lanes_log2) < chunks) ++t.lanes_log2;
    const int piece = Chunks << t.lanes_log2, at_once = kThreads >> t.lanes_log2;
    t.pieces = (uint32_t)((chunks + piece - 1) / piece);
    t.units = (rows + at_once - 1) / at_once * t.pieces;
    return t;
}
int grid_of(int64_t units) { return (int)std::min<int64_t>(units, 1 << 20); }

// ---- forward

constexpr int kEmbedChunks = 2;

template <typename T, bool Whole>
__global__ __launch_bounds__(kThreads) void k_embed(EmbedParams p, SeqLengths lens, Tiles tiles)
{
    using Store = typename T::Store;
    const int lanes = 1 << tiles.lanes_log2, lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> tiles.lanes_log2;
    const uint32_t rows = (uint32_t)p.B * (uint32_t)p.T;
    const int at_once = kThreads >> tiles.lanes_log2, chunks = (p.D + 7) / 8;
    for (int64_t u = blockIdx.x; u < tiles.units; u += gridDim.x) {
        const uint32_t group = (uint32_t)(u / tiles.pieces), piece = (uint32_t)(u - (int64_t)group * tiles.pieces);
        const uint32_t row = group * (uint32_t)at_once + sub;
        if (row >= rows) continue;
        int64_t token = inside(lens, row, p.T) ? token_at(p.tokens, p.token_bytes, row) : -1;
        const bool bad = token >= p.V;
        const int first = (int)piece * kEmbedChunks * lanes + lane;
        if (p.status && first == 0) p.status[row] = bad ? 4 : 0;
        float f[kEmbedChunks][8];
#pragma unroll
        for (int k = 0; k < kEmbedChunks; ++k) {
            const int c = first + k * lanes;
#pragma unroll
            for (int i = 0; i < 8; ++i) f[k][i] = bad ? NAN : 0.f;
            if (c < chunks && !bad && token >= 0)
                load_at<T, Whole>(static_cast<const Store*>(p.table) + token * p.stride, c, p.D, f[k]);
        }
#pragma unroll
        for (int k = 0; k < kEmbedChunks; ++k) {
            const int c = first + k * lanes;
            if (c >= chunks) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) f[k][i] = token < 0 ? 0.f : f[k][i] * p.scale;
            store_at<T, Whole>(static_cast<Store*>(p.out) + (int64_t)row * p.D, c, p.D, f[k]);
        }
    }
}

// ---- sorting positions by token: digits of p.plan.bits bits, the lowest first, every pass keeps the order of
// equal digits. Keys are tokens; V where there is none, or none of the table.

// (the counters of frequent tokens and pieces are cleared on the way)
__global__ __launch_bounds__(kThreads) void k_embed_keys(EmbedGradParams p, SeqLengths lens, uint32_t from, uint32_t n,
                                                         uint32_t* keys, uint32_t* counts)
{
    if (from == 0 && blockIdx.x == 0 && threadIdx.x < 2) counts[threadIdx.x] = 0;
    for (uint32_t i = blockIdx.x * kThreads + threadIdx.x; i < n; i += gridDim.x * kThreads) {
        const int64_t token = inside(lens, i, p.T) ? token_at(p.tokens, p.token_bytes, from + i) : -1;
        keys[from + i] = token < 0 || token >= p.V ? (uint32_t)p.V : (uint32_t)token;
    }
}

// How many keys of every tile have a digit: hist[digit][tile].
__global__ __launch_bounds__(kThreads) void k_embed_count(const uint32_t* keys, uint32_t N, int shift, int bits,
                                                          uint32_t tiles, uint32_t* hist)
{
    extern __shared__ uint32_t bins[];
    const int n = 1 << bits;
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        for (int i = threadIdx.x; i < n; i += kThreads) bins[i] = 0;
        __syncthreads();
        for (int k = 0; k < kEmbedTile / kThreads; ++k) {
            const uint32_t i = tile * kEmbedTile + k * kThreads + threadIdx.x;
            if (i < N) atomicAdd(&bins[keys[i] >> shift & (n - 1)], 1u);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kThreads) hist[(int64_t)i * tiles + tile] = bins[i];
        __syncthreads();
    }
}

// Sums of all entries before each, by one workgroup.
constexpr int kScanThreads = 1024;
__global__ __launch_bounds__(kScanThreads) void k_embed_scan(uint32_t* hist, int64_t n)
{
    __shared__ uint32_t sums[2][kScanThreads];
    const int64_t each = (n + kScanThreads - 1) / kScanThreads;
    const int64_t from = min(n, each * threadIdx.x), to = min(n, from + each);
    uint32_t s = 0;
    for (int64_t i = from; i < to; ++i) s += hist[i];
    int now = 0;
    sums[0][threadIdx.x] = s;
    __syncthreads();
    for (int o = 1; o < kScanThreads; o <<= 1) {
        uint32_t v = sums[now][threadIdx.x];
        if ((int)threadIdx.x >= o) v += sums[now][threadIdx.x - o];
        sums[now ^ 1][threadIdx.x] = v;
        now ^= 1;
        __syncthreads();
    }
    uint32_t before = threadIdx.x > 0 ? sums[now][threadIdx.x - 1] : 0;
    for (int64_t i = from; i < to; ++i) {
        const uint32_t v = hist[i];
        hist[i] = before;
        before += v;
    }
}

// Keys of a tile to their places. A wave takes a quarter of the tile, 64 keys at a time in order; lanes with equal
// digits find each other by a ballot on each bit.
__global__ __launch_bounds__(kThreads) void k_embed_place(const uint32_t* keys, const uint32_t* order, uint32_t N,
                                                          int shift, int bits, uint32_t tiles, const uint32_t* hist,
                                                          uint32_t* keys_out, uint32_t* order_out)
{
    extern __shared__ uint32_t places[];  // [wave][digit]
    const int n = 1 << bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int kStrips = kEmbedTile / kThreads;
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        for (int i = threadIdx.x; i < n * kWaves; i += kThreads) places[i] = 0;
        __syncthreads();
        const uint32_t first = tile * kEmbedTile + wave * (kEmbedTile / kWaves) + lane;
        uint32_t key[kStrips], from[kStrips];
#pragma unroll
        for (int k = 0; k < kStrips; ++k) {
            const uint32_t i = first + k * 64;
            key[k] = i < N ? keys[i] : 0;
            from[k] = i < N ? (order ? order[i] : i) : 0;
            if (i < N) atomicAdd(&places[wave * n + (key[k] >> shift & (n - 1))], 1u);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kThreads) {
            uint32_t at = hist[(int64_t)i * tiles + tile];
            for (int w = 0; w < kWaves; ++w) {
                const uint32_t count = places[w * n + i];
                places[w * n + i] = at;
                at += count;
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kStrips; ++k) {
            const bool here = first + k * 64 < N;
            const uint32_t digit = key[k] >> shift & (n - 1);
            uint64_t same = __ballot(here);
            for (int b = 0; b < bits; ++b) {
                const bool bit = digit >> b & 1;
                const uint64_t set = __ballot(bit);
                same &= bit ? set : ~set;
            }
            volatile uint32_t* place = &places[wave * n + digit];
            uint32_t at = 0;
            if (here) at = *place + __popcll(same & ((1ull << lane) - 1));
            __builtin_amdgcn_wave_barrier();
            if (here && (same >> lane) == 1) *place = at + 1;  // the last of them
            __builtin_amdgcn_wave_barrier();
            if (here) {
                keys_out[at] = key[k];
                order_out[at] = from[k];
            }
        }
        __syncthreads();
    }
}

__device__ __forceinline__ uint32_t lower_bound(const uint32_t* keys, uint32_t n, uint32_t key)
{
    uint32_t lo = 0, hi = n;
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (keys[mid] < key) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// Where the positions of every token begin, and pieces of those of frequent ones. Which numbers a token's pieces get is
// left to chance; they go by those numbers alone.
__global__ __launch_bounds__(kThreads) void k_embed_starts(const uint32_t* keys, uint32_t N, int V, uint32_t* starts,
                                                           uint32_t* counts, uint2* first, uint2* piece)
{
    for (int64_t v = (int64_t)blockIdx.x * kThreads + threadIdx.x; v <= V; v += (int64_t)gridDim.x * kThreads) {
        const uint32_t at = lower_bound(keys, N, (uint32_t)v);
        starts[v] = at;
        if (v == V) continue;
        const uint32_t count = lower_bound(keys, N, (uint32_t)v + 1) - at;
        if (count <= kEmbedPiece) continue;
        const uint32_t n = (count + kEmbedPiece - 1) / kEmbedPiece;
        const uint32_t k = atomicAdd(&counts[0], 1u), to = atomicAdd(&counts[1], n);
        first[k] = make_uint2((uint32_t)v, to);
        for (uint32_t i = 0; i < n; ++i)
            piece[to + i] = make_uint2(at + i * kEmbedPiece, min((uint32_t)kEmbedPiece, count - i * kEmbedPiece));
    }
}

// ---- sums of rows

// Adds the chunk of positions order[from..from + n - 1] up, in that order.
template <typename T, bool Whole>
__device__ __forceinline__ void add_rows(const EmbedGradParams& p, const uint32_t* order, uint32_t from, uint32_t n,
                                         int c, float* s)
{
    using Store = typename T::Store;
    constexpr int kAtOnce = 4;
    const Store* g = static_cast<const Store*>(p.g);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = 0.f;
    for (uint32_t k = 0; k < n; k += kAtOnce) {
        Raw<T> v[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const uint32_t pos = order[from + min(k + j, n - 1)], b = pos / (uint32_t)p.T;
            v[j] = raw_at<T, Whole>(g + (int64_t)b * p.stride_b + (int64_t)(pos - b * (uint32_t)p.T) * p.stride_t, c, p.D);
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (k + j >= n) continue;
            float f[8];
            unpack_at<T, Whole>(v[j], c, p.D, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += f[i];
        }
    }
}

template <typename T, bool Whole>
__device__ __forceinline__ void write_grad(const EmbedGradParams& p, uint32_t v, int c, const float* s)
{
    typename T::Store* out = static_cast<typename T::Store*>(p.grad) + (int64_t)v * p.D;
    float f[8];
    if (p.accumulate) load_at<T, Whole>(out, c, p.D, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = p.accumulate ? f[i] + s[i] * p.scale : s[i] * p.scale;
    store_at<T, Whole>(out, c, p.D, f);
}

// Rows of the table with at most kEmbedPiece positions, those with none among them.
template <typename T, bool Whole>
__global__ __launch_bounds__(kThreads) void k_embed_rows(EmbedGradParams p, Tiles tiles, const uint32_t* starts,
                                                         const uint32_t* order)
{
    const int lanes = 1 << tiles.lanes_log2, lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> tiles.lanes_log2;
    const int at_once = kThreads >> tiles.lanes_log2, chunks = (p.D + 7) / 8;
    for (int64_t u = blockIdx.x; u < tiles.units; u += gridDim.x) {
        const int64_t group = u / tiles.pieces, v = group * at_once + sub;
        const int c = (int)(u - group * tiles.pieces) * lanes + lane;
        if (v >= p.V || c >= chunks) continue;
        const uint32_t from = starts[v], n = starts[v + 1] - from;
        if (n > kEmbedPiece || (n == 0 && p.accumulate)) continue;
        float s[8];
        add_rows<T, Whole>(p, order, from, n, c, s);
        write_grad<T, Whole>(p, (uint32_t)v, c, s);
    }
}

template <typename T, bool Whole>
__global__ __launch_bounds__(kThreads) void k_embed_pieces(EmbedGradParams p, Tiles tiles, const uint32_t* counts,
                                                           const uint2* piece, const uint32_t* order, float* partials)
{
    const int lanes = 1 << tiles.lanes_log2, lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> tiles.lanes_log2;
    const int at_once = kThreads >> tiles.lanes_log2, chunks = (p.D + 7) / 8;
    const uint32_t n = counts[1];
    for (int64_t u = blockIdx.x; u < tiles.units; u += gridDim.x) {
        const int64_t group = u / tiles.pieces, k = group * at_once + sub;
        const int c = (int)(u - group * tiles.pieces) * lanes + lane;
        if (k >= n || c >= chunks) continue;
        const uint2 q = piece[k];
        float s[8];
        add_rows<T, Whole>(p, order, q.x, q.y, c, s);
        store_at<F32, Whole>(partials + k * p.D, c, p.D, s);
    }
}

// Frequent tokens, from their pieces.
template <typename T, bool Whole>
__global__ __launch_bounds__(kThreads) void k_embed_join(EmbedGradParams p, Tiles tiles, const uint32_t* counts,
                                                         const uint2* first, const uint32_t* starts,
                                                         const float* partials)
{
    const int lanes = 1 << tiles.lanes_log2, lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> tiles.lanes_log2;
    const int at_once = kThreads >> tiles.lanes_log2, chunks = (p.D + 7) / 8;
    const uint32_t heavy = counts[0];
    for (int64_t u = blockIdx.x; u < tiles.units; u += gridDim.x) {
        const int64_t group = u / tiles.pieces, k = group * at_once + sub;
        const int c = (int)(u - group * tiles.pieces) * lanes + lane;
        if (k >= heavy || c >= chunks) continue;
        const uint32_t v = first[k].x, n = (starts[v + 1] - starts[v] + kEmbedPiece - 1) / kEmbedPiece;
        const float* part = partials + (int64_t)first[k].y * p.D;
        float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (uint32_t i = 0; i < n; ++i) {
            float f[8];
            load_at<F32, Whole>(part + (int64_t)i * p.D, c, p.D, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] += f[j];
        }
        write_grad<T, Whole>(p, v, c, s);
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
    const Tiles t = tiles_of<kEmbedChunks>((int64_t)p.B * p.T, p.D);
    by_type(dtype, [&](auto type) {
        by_whole(p.D, [&](auto whole) {
            k_embed<decltype(type), decltype(whole)::value><<<grid_of(t.units), kThreads, 0, stream>>>(p, lens, t);
        });
    });
    return hipGetLastError();
}

EmbedPlan plan_embed(int64_t N, int V, int D)
{
    EmbedPlan p{};
    int bits = 1;  // of a key: V is one
    while (bits < 31 && (int64_t)V >> bits > 0) ++bits;
    p.passes = (bits + 9) / 10;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.tiles = (int32_t)((N + kEmbedTile - 1) / kEmbedTile);
    // a frequent token has kEmbedPiece + 1 positions or more, all its pieces but the last are full
    p.heavy = (int32_t)(N / (kEmbedPiece + 1));
    p.pieces = (int32_t)(N / kEmbedPiece + p.heavy);
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
    p.counts = take(8);
    p.first = take((size_t)p.heavy * 8);
    p.piece = take((size_t)p.pieces * 8);
    p.partials = take((size_t)p.pieces * D * 4);
    p.bytes = at;
    return p;
}

hipError_t launch_embed_keys(const EmbedGradParams& p, const SeqLengths& lens, int b, int n, hipStream_t stream)
{
    const uint32_t count = (uint32_t)n * (uint32_t)p.T;
    const int grid = (int)std::min<int64_t>(((int64_t)count + kThreads - 1) / kThreads, 4096);
    k_embed_keys<<<grid, kThreads, 0, stream>>>(p, lens, (uint32_t)b * (uint32_t)p.T, count,
                                                place<uint32_t>(p, p.plan.keys), place<uint32_t>(p, p.plan.counts));
    return hipGetLastError();
}

hipError_t launch_embed_grad(const EmbedGradParams& p, int dtype, hipStream_t stream)
{
    const EmbedPlan& plan = p.plan;
    const uint32_t N = (uint32_t)p.B * (uint32_t)p.T;
    uint32_t* keys[2] = {place<uint32_t>(p, plan.keys), place<uint32_t>(p, plan.keys) + N};
    uint32_t* order[2] = {place<uint32_t>(p, plan.order), place<uint32_t>(p, plan.order) + N};
    uint32_t* hist = place<uint32_t>(p, plan.hist);
    uint32_t* starts = place<uint32_t>(p, plan.starts);
    uint32_t* counts = place<uint32_t>(p, plan.counts);
    uint2* first = place<uint2>(p, plan.first);
    uint2* piece = place<uint2>(p, plan.piece);
    float* partials = place<float>(p, plan.partials);
    int now = 0;
    const int grid = std::min(plan.tiles, 1 << 16);
    const int bins = 4 << plan.bits;
    for (int pass = 0; N > 0 && pass < plan.passes; ++pass, now ^= 1) {
        const int shift = pass * plan.bits;
        k_embed_count<<<grid, kThreads, bins, stream>>>(keys[now], N, shift, plan.bits, plan.tiles, hist);
        k_embed_scan<<<1, kScanThreads, 0, stream>>>(hist, (int64_t)plan.tiles << plan.bits);
        k_embed_place<<<grid, kThreads, bins * kWaves, stream>>>(keys[now], pass ? order[now] : nullptr, N, shift,
                                                                 plan.bits, plan.tiles, hist, keys[now ^ 1],
                                                                 order[now ^ 1]);
    }
    const int64_t v = ((int64_t)p.V + 1 + kThreads - 1) / kThreads;
    k_embed_starts<<<grid_of(v), kThreads, 0, stream>>>(keys[now], N, p.V, starts, counts, first, piece);
    const Tiles rows = tiles_of<1>(p.V, p.D);
    by_type(dtype, [&](auto type) {
        by_whole(p.D, [&](auto whole) {
            using T = decltype(type);
            constexpr bool kWhole = decltype(whole)::value;
            k_embed_rows<T, kWhole><<<grid_of(rows.units), kThreads, 0, stream>>>(p, rows, starts, order[now]);
            if (plan.heavy == 0) return;
            const Tiles pieces = tiles_of<1>(plan.pieces, p.D), heavy = tiles_of<1>(plan.heavy, p.D);
            k_embed_pieces<T, kWhole>
                <<<grid_of(pieces.units), kThreads, 0, stream>>>(p, pieces, counts, piece, order[now], partials);
            k_embed_join<T, kWhole>
                <<<grid_of(heavy.units), kThreads, 0, stream>>>(p, heavy, counts, first, starts, partials);
        });
    });
    return hipGetLastError();
}

}  // namespace lfmmi
