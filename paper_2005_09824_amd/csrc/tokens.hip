// Log probabilities of given tokens, with entropy and the best alternatives of every row of
// logits, and their gradient. See include/lfmmi.h for the formulas.
#include <hip/hip_runtime.h>

#include "../../include/lfmmi.h"
#include "operators.h"
#include "vec16.h"

namespace lfmmi {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.693147180559945309f;
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kLoads = 4;  // 16-byte loads that a lane has in flight

// 2^y as the hardware has it: results below the normal range are 0, which sums beside 1
// do not notice.
__device__ __forceinline__ float exp2_of(float y) { return __builtin_amdgcn_exp2f(y); }

// (fmaxf quiets its operands first, an instruction for each; a NaN shows in the sums whatever
// this makes of it)
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// ---- reductions over G lanes: 16 (a DPP row) or 64 (a wave); every lane has the result

template <int Ror>
__device__ __forceinline__ float rotated(float v)
{
    const int i = __float_as_int(v);
    return __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x120 + Ror, 0xf, 0xf, true));
}
__device__ __forceinline__ float lane_of(float v, int lane)
{
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
template <int G>
__device__ __forceinline__ float sum_over(float v)
{
    v += rotated<8>(v);
    v += rotated<4>(v);
    v += rotated<2>(v);
    v += rotated<1>(v);
    if (G == 64) v = (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
    return v;
}
template <int G>
__device__ __forceinline__ float max_over(float v)
{
    v = fmaxf(v, rotated<8>(v));
    v = fmaxf(v, rotated<4>(v));
    v = fmaxf(v, rotated<2>(v));
    v = fmaxf(v, rotated<1>(v));
    if (G == 64) v = fmaxf(fmaxf(lane_of(v, 0), lane_of(v, 16)), fmaxf(lane_of(v, 32), lane_of(v, 48)));
    return v;
}

// What a lane, a wave and a workgroup know of the logits they have read: the largest of them,
// and over all of them, with y = (x - m) * scale * log2(e), the sums of 2^y and of y 2^y.
// The entropy comes from the second sum without cancellation: ln s and -y are both >= 0.
struct Sums {
    float m, s, u;
};

// m starts at the lowest finite value, not at -inf: differences to it are then never
// (-inf) - (-inf), and a row of nothing but -inf ends with s == 0. A row of nothing but the
// type's lowest value is a uniform one.
__device__ __forceinline__ Sums no_sums() { return {-3.402823466e38f, 0.f, 0.f}; }

// (y may be -inf, from a mask or a difference that overflows: clamped where 0 * y is meant to
// be 0; a NaN stays in 2^y)
__device__ __forceinline__ float finite(float y) { return fmaxf(y, -1e30f); }

// Sums taken against m, as they are against `to` >= m.
__device__ __forceinline__ void shift(Sums& a, float to, float scale2)
{
    const float dy = finite((a.m - to) * scale2);
    const float f = exp2_of(dy);
    a.u = f * (a.u + dy * a.s);
    a.s *= f;
    a.m = to;
}

template <int G>
__device__ __forceinline__ void join_lanes(Sums& a, float scale2)
{
    shift(a, max_over<G>(a.m), scale2);
    a.s = sum_over<G>(a.s);
    a.u = sum_over<G>(a.u);
}

template <bool Ent>
__device__ __forceinline__ void add(Sums& a, float x, float scale2)
{
    const float y = (x - a.m) * scale2, e = exp2_of(y);
    a.s += e;
    if (Ent) a.u += e * finite(y);
}

// Values in an order of whole numbers, equal ones (-0 and 0 are) by index, lowest first. No
// value has key 0.
__device__ __forceinline__ uint64_t key_of(float x, int i)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    const uint32_t v = b >> 31 ? ~b : b | 0x80000000u;
    return (uint64_t)v << 32 | (uint32_t)~i;
}
__device__ __forceinline__ int index_of(uint64_t key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ float value_of(uint64_t key)
{
    const uint32_t v = (uint32_t)(key >> 32);
    return __uint_as_float(v >> 31 ? v & 0x7fffffffu : ~v);
}

struct Row {
    bool live;
    int64_t target;  // -1: none given
};

template <typename P>
__device__ __forceinline__ Row row_of(const P& p, const SeqLengths& lens, int b, int t)
{
    Row r{true, -1};
    if (lens.n > 0 && t >= lens.T[b]) return {false, -1};
    if (p.targets) {
        const int64_t at = (int64_t)b * p.T + t;
        r.target = p.target_bytes == 8 ? static_cast<const int64_t*>(p.targets)[at]
                                       : static_cast<const int32_t*>(p.targets)[at];
        r.live = r.target >= 0;
    }
    return r;
}

// What a row's alternatives need to know of it. m: NaN for a row with a NaN or +inf logit,
// -inf for one of nothing but -inf.
struct Scores {
    float m, logs;
};

// The flags in a row's sums: 2, 1 or 0.
__device__ __forceinline__ int flags_of(const Sums& a)
{
    return !(a.s < INFINITY) ? 2 : a.s == 0.f ? 1 : 0;  // (NaN, or an inf - inf on the way: 2)
}

__device__ __forceinline__ Scores scores_of(const Sums& a)
{
    const int flags = flags_of(a);
    const float bad = flags == 2 ? NAN : -INFINITY;
    return flags ? Scores{bad, bad} : Scores{a.m, log2f(a.s) * kLn2};
}

// Everything but the alternatives, by one lane.
__device__ __forceinline__ void write_row(const TokenParams& p, int64_t row, const Row& r, const Sums& a,
                                          float x_target)
{
    int flags = 0;
    float logp = 0.f, entropy = 0.f;
    Scores c{0.f, 0.f};
    if (r.live) {
        flags = flags_of(a);
        c = scores_of(a);
        entropy = flags == 2 ? NAN : flags == 1 ? 0.f : c.logs - kLn2 * (a.u / a.s);
        logp = flags ? c.m : (x_target - c.m) * p.scale - c.logs;
        if (r.target >= p.V) {
            flags |= 4;
            logp = NAN;
        }
    }
    if (p.logp) p.logp[row] = logp;
    if (p.entropy) p.entropy[row] = entropy;
    if (p.stats) {
        p.stats[2 * row] = c.m;
        p.stats[2 * row + 1] = c.logs;
    }
    if (p.status) p.status[row] = flags;
}

// (of a row that is not scored: live false)
__device__ __forceinline__ void write_top(const TokenParams& p, int64_t row, int k, uint64_t key, bool live,
                                          Scores c)
{
    const int64_t at = row * p.top_k + k;
    if (p.top_id) p.top_id[at] = live && !(c.m != c.m) ? index_of(key) : -1;
    if (p.top_logp)
        p.top_logp[at] =
            !live ? 0.f : c.m == -INFINITY ? -INFINITY : (value_of(key) - c.m) * p.scale - c.logs;
}

// ---- one pass over n logits by G lanes

// Chunks of 16 bytes go round the lanes; a lane takes kLoads of them at a time. `best` is the
// largest value a lane met in whole chunks (-inf to begin with), `best_at` the first group of
// kLoads chunks that held it.
struct Best {
    float value;
    int group;
};

template <typename D, int G>
__device__ __forceinline__ void load_group(const typename D::Store* x, int full, int q, uint4* r)
{
    if (__builtin_expect(q - (q & (G - 1)) + kLoads * G <= full, 1)) {
#pragma unroll
        for (int k = 0; k < kLoads; ++k) r[k] = load16(x + (int64_t)(q + k * G) * D::kVec);
    } else {
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            r[k] = make_uint4(D::kNone, D::kNone, D::kNone, D::kNone);
            if (q + k * G < full) r[k] = load16(x + (int64_t)(q + k * G) * D::kVec);
        }
    }
}

// Per logit of 16 bits: half an instruction for the maximum, one to unpack it, two for y, four
// issue slots for 2^y, one for each sum and one for the clamp.
template <typename D, int G, bool Ent, bool Top>
__device__ __forceinline__ void scan(const typename D::Store* x, int n, int lane, float scale2, Sums& a,
                                     Best& best)
{
    constexpr int N = D::kVec * kLoads;
    const int full = n / D::kVec;
    for (int q = lane, j = 0; q - lane < full; q += kLoads * G, ++j) {
        uint4 r[kLoads];
        load_group<D, G>(x, full, q, r);
        float f[N];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) D::unpack(r[k], f + k * D::kVec);
        float top = max3(f[0], f[1], f[2]);
#pragma unroll
        for (int i = 3; i + 1 < N; i += 2) top = max3(top, f[i], f[i + 1]);
        if (N % 2 == 0) top = max3(top, f[N - 1], f[N - 1]);
        if (Top && top > best.value) best = {top, j};
        shift(a, fmaxf(a.m, top), scale2);
        float s[4] = {a.s, 0.f, 0.f, 0.f}, u[4] = {a.u, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = (f[i] - a.m) * scale2, e = exp2_of(y);
            s[i & 3] += e;
            if (Ent) u[i & 3] += e * finite(y);
        }
        a.s = (s[0] + s[1]) + (s[2] + s[3]);
        a.u = (u[0] + u[1]) + (u[2] + u[3]);
    }
    for (int i = full * D::kVec + lane; i < n; i += G) {
        const float v = D::load(x + i);
        shift(a, fmaxf(a.m, v), scale2);
        add<Ent>(a, v, scale2);
    }
}

// ---- the best alternatives
//
// The k-th largest of the lanes' own largest keys is a lower bound T of the k-th largest key
// of the row, and every key from T on lies with one of the k lanes whose own largest is from T
// on. So one pass finds a lane's largest value, and only k lanes' logits are looked at
// again, from the cache, by all lanes together; rarely many more than k of them reach T. Those
// are put in order by counting, for each, how many are larger.

// The key of a lane's largest value in whole chunks: the group that held it is read again for the
// lowest index. 0 for a lane that had no chunk.
template <typename D, int G>
__device__ __forceinline__ uint64_t best_key(const typename D::Store* x, int n, int lane, const Best& best,
                                             int offset)
{
    const int full = n / D::kVec;
    if (lane >= full) return 0;
    const int q = best.group * kLoads * G + lane;
    int at = 0;
#pragma unroll
    for (int k = kLoads - 1; k >= 0; --k) {
        if (q + k * G >= full) continue;
        float f[D::kVec];
        D::unpack(load16(x + (int64_t)(q + k * G) * D::kVec), f);
#pragma unroll
        for (int i = D::kVec - 1; i >= 0; --i)
            if (f[i] == best.value) at = (q + k * G) * D::kVec + i;
    }
    return key_of(best.value, offset + at);
}

// By a wave whose lanes hold N keys each: the k-th largest of the keys that are not 0 (keys are
// different but for 0), or a lower bound of it with no key between; 0 if there are fewer.
template <int N>
__device__ __forceinline__ uint64_t kth_key(const uint64_t (&key)[N], int k)
{
    uint64_t t = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t c = t | (uint64_t)1 << bit;
        int count = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) count += __popcll(__ballot(key[i] >= c));
        if (count >= k) t = c;
        if (count == k) break;
    }
    return t;
}

// LDS of one row's selection.
template <int G>
struct Selection {
    static constexpr int kCap = G == 64 ? 512 : 1024;  // keys from T on that it holds
    uint64_t list[kCap];
    int lanes[kMaxTop];
    int num_lanes, count;
    uint64_t from;  // T
};

template <int G>
__device__ __forceinline__ void row_sync()
{
    if (G == 64) {  // one wave: its LDS operations are carried out in order
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    } else {
        __syncthreads();
    }
}

template <int G>
__device__ __forceinline__ void push(Selection<G>& sel, uint64_t key)
{
    const int at = atomicAdd(&sel.count, 1);
    if (at < Selection<G>::kCap) sel.list[at] = key;
}

// From T and the lanes that reach it to the list of all keys that do.
template <typename D, int G>
__device__ __forceinline__ void gather(const typename D::Store* x, int n, int lane, int offset, Selection<G>& sel)
{
    const int full = n / D::kVec, lanes = sel.num_lanes;
    const uint64_t from = sel.from;
    // (T need not be a key: below that of -inf its bits are no number's)
    const float least = (uint32_t)(from >> 32) <= 0x007fffffu ? -INFINITY : value_of(from);
    const int deep = (full + G - 1) / G;  // chunks a lane has at most
    for (int w = lane; w < lanes * deep; w += G) {
        const int q = w / lanes * G + sel.lanes[w % lanes];
        if (q >= full) continue;
        float f[D::kVec];
        D::unpack(load16(x + (int64_t)q * D::kVec), f);
#pragma unroll
        for (int i = 0; i < D::kVec; ++i)
            if (f[i] >= least) {
                const uint64_t key = key_of(f[i], offset + q * D::kVec + i);
                if (key >= from) push(sel, key);
            }
    }
    for (int i = full * D::kVec + lane; i < n; i += G) {
        const uint64_t key = key_of(D::load(x + i), offset + i);
        if (key >= from) push(sel, key);
    }
}

// The k best of n logits, handed to put(rank, key) by the lane that has one. Key indices start at
// `offset`. `mine`: this lane's best_key.
template <typename D, int G, typename Put>
__device__ __forceinline__ void select_top(const typename D::Store* x, int n, int lane, int offset, int k,
                                           uint64_t mine, Selection<G>& sel, Put&& put)
{
    if (G == 64) {
        const uint64_t keys[1] = {mine};
        const uint64_t from = kth_key(keys, k);
        const bool in = mine != 0 && mine >= from;
        const uint64_t mask = __ballot(in);
        if (in) sel.lanes[__popcll(mask & (((uint64_t)1 << lane) - 1))] = lane;
        if (lane == 0) {
            sel.num_lanes = __popcll(mask);
            sel.count = 0;
            sel.from = from;
        }
    } else {
        sel.list[lane] = mine;
        __syncthreads();
        if (lane < 64) {
            const uint64_t keys[4] = {sel.list[lane], sel.list[lane + 64], sel.list[lane + 128],
                                      sel.list[lane + 192]};
            const uint64_t from = kth_key(keys, k);
            int base = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = keys[i] != 0 && keys[i] >= from;
                const uint64_t mask = __ballot(in);
                if (in) sel.lanes[base + __popcll(mask & (((uint64_t)1 << lane) - 1))] = lane + 64 * i;
                base += __popcll(mask);
            }
            if (lane == 0) {
                sel.num_lanes = base;
                sel.count = 0;
                sel.from = from;
            }
        }
    }
    row_sync<G>();
    gather<D, G>(x, n, lane, offset, sel);
    row_sync<G>();
    const int count = sel.count;
    if (__builtin_expect(count <= Selection<G>::kCap, 1)) {
        for (int i = lane; i < count; i += G) {
            const uint64_t key = sel.list[i];
            int rank = 0;
            for (int j = 0; j < count; ++j) rank += sel.list[j] > key;
            if (rank < k) put(rank, key);
        }
        return;
    }
    // k or fewer lanes hold more large values than the list does: one pass for each alternative
    uint64_t last = ~(uint64_t)0;
    for (int rank = 0; rank < k; ++rank) {
        uint64_t top = 0;
        for (int i = lane; i < n; i += G) {
            const uint64_t key = key_of(D::load(x + i), offset + i);
            if (key < last && key > top) top = key;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const uint64_t other = __shfl_xor(top, o, 64);
            top = other > top ? other : top;
        }
        if (G > 64) {
            row_sync<G>();
            if ((lane & 63) == 0) sel.list[lane >> 6] = top;
            row_sync<G>();
            for (int w = 0; w < G / 64; ++w) top = sel.list[w] > top ? sel.list[w] : top;
        }
        if (lane == 0) put(rank, top);
        last = top;
    }
}

// ---- forward kernels

template <typename P>
__device__ __forceinline__ const void* row_at(const P& p, int b, int t, size_t size)
{
    return static_cast<const char*>(p.x) + (b * p.stride_b + t * p.stride_t) * (int64_t)size;
}

// G = 16 or 64 lanes a row, kThreads / G rows a workgroup.
template <typename D, int G, bool Ent, bool Top>
__global__ __launch_bounds__(kThreads) void k_token_rows(TokenParams p, SeqLengths lens)
{
    static_assert(!Top || G == 64, "a selection takes a wave");
    using Store = typename D::Store;
    constexpr int kRows = kThreads / G;
    __shared__ Selection<64> sels[Top ? kWaves : 1];
    const int lane = threadIdx.x % G, sub = threadIdx.x / G;
    const float scale2 = p.scale * kLog2e;
    const uint32_t rows = (uint32_t)p.B * p.T;  // (below 2^31: sums with a grid fit 32 bits)
    for (uint32_t row = blockIdx.x * kRows + sub; row < rows; row += gridDim.x * kRows) {
        const int b = row / p.T, t = row % p.T;
        const Row r = row_of(p, lens, b, t);
        const Store* x = static_cast<const Store*>(row_at(p, b, t, sizeof(Store)));
        Sums a = no_sums();
        Best best{-INFINITY, 0};
        float xt = 0.f;
        if (r.live) {
            if (r.target >= 0 && r.target < p.V) xt = D::load(x + r.target);
            scan<D, G, Ent, Top>(x, p.V, lane, scale2, a, best);
            join_lanes<G>(a, scale2);
        }
        if (lane == 0) write_row(p, row, r, a, xt);
        if (!Top) continue;
        const Scores c = scores_of(a);
        if (!r.live || c.m != c.m) {
            for (int k = lane; k < p.top_k; k += G) write_top(p, row, k, 0, r.live, c);
        } else {
            const uint64_t mine = best_key<D, G>(x, p.V, lane, best, 0);
            select_top<D, 64>(x, p.V, lane, 0, p.top_k, mine, sels[sub % kWaves],
                              [&](int k, uint64_t key) { write_top(p, row, k, key, true, c); });
            row_sync<64>();
        }
    }
}

// What part j of `parts` of a row leaves for k_token_join: sums, and its k best keys.
__device__ __forceinline__ float4* part_sums(const TokenParams& p, int64_t part)
{
    return static_cast<float4*>(p.workspace) + part;
}
__device__ __forceinline__ uint64_t* part_keys(const TokenParams& p, int64_t part)
{
    const int64_t all = (int64_t)p.B * p.T * p.parts;
    return reinterpret_cast<uint64_t*>(part_sums(p, all)) + part * p.top_k;
}

// The workgroup's sums from its lanes'; every lane has them.
__device__ __forceinline__ Sums join_waves(Sums a, float scale2, Sums* shared)
{
    join_lanes<64>(a, scale2);
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = a;
    __syncthreads();
    a = shared[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        Sums o = shared[w];
        const float to = fmaxf(a.m, o.m);
        shift(a, to, scale2);
        shift(o, to, scale2);
        a.s += o.s;
        a.u += o.u;
    }
    return a;
}

// A workgroup a row, or for Split a workgroup for each of p.parts parts of a row.
template <typename D, bool Ent, bool Top, bool Split>
__global__ __launch_bounds__(kThreads) void k_token_blocks(TokenParams p, SeqLengths lens)
{
    using Store = typename D::Store;
    __shared__ Sums shared[kWaves];
    __shared__ Selection<kThreads> sel;
    const int lane = threadIdx.x;
    const float scale2 = p.scale * kLog2e;
    // (rows of several parts are few)
    const uint32_t units = (uint32_t)p.B * p.T * (Split ? p.parts : 1);
    for (uint32_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const uint32_t row = Split ? unit / p.parts : unit;
        const int from = Split ? (int)(unit % p.parts) * p.part_size : 0;
        const int n = Split ? (p.V - from < p.part_size ? p.V - from : p.part_size) : p.V;
        const int b = row / p.T, t = row % p.T;
        const Row r = row_of(p, lens, b, t);
        const Store* x = static_cast<const Store*>(row_at(p, b, t, sizeof(Store))) + from;
        Sums a = no_sums();
        Best best{-INFINITY, 0};
        float xt = 0.f;
        if (r.live) {
            if (!Split && r.target >= 0 && r.target < p.V) xt = D::load(x + r.target);
            scan<D, kThreads, Ent, Top>(x, n, lane, scale2, a, best);
            a = join_waves(a, scale2, shared);
        }
        if (lane == 0) {
            if (!Split) write_row(p, row, r, a, xt);
            else if (r.live) *part_sums(p, unit) = make_float4(a.m, a.s, a.u, 0.f);
        }
        if (Top && (Split ? r.live : true)) {
            const Scores c = scores_of(a);
            if (!r.live || c.m != c.m) {
                for (int k = lane; k < p.top_k; k += kThreads) {
                    if (Split) part_keys(p, unit)[k] = 0;
                    else write_top(p, row, k, 0, r.live, c);
                }
            } else {
                const uint64_t mine = best_key<D, kThreads>(x, n, lane, best, from);
                const int k = p.top_k < n ? p.top_k : n;
                select_top<D, kThreads>(x, n, lane, from, k, mine, sel, [&](int rank, uint64_t key) {
                    if (Split) part_keys(p, unit)[rank] = key;
                    else write_top(p, row, rank, key, true, c);
                });
                if (Split)
                    for (int rank = k + lane; rank < p.top_k; rank += kThreads) part_keys(p, unit)[rank] = 0;
            }
        }
        __syncthreads();
    }
}

// A workgroup a row: joins the parts' sums and alternatives.
template <typename D, bool Top>
__global__ __launch_bounds__(kThreads) void k_token_join(TokenParams p, SeqLengths lens)
{
    using Store = typename D::Store;
    __shared__ Sums shared[kWaves];
    __shared__ Selection<kThreads> sel;
    const int lane = threadIdx.x;
    const float scale2 = p.scale * kLog2e;
    const uint32_t rows = (uint32_t)p.B * p.T;
    for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const int b = row / p.T, t = row % p.T;
        const Row r = row_of(p, lens, b, t);
        const Store* x = static_cast<const Store*>(row_at(p, b, t, sizeof(Store)));
        Sums a = no_sums();
        float xt = 0.f;
        uint64_t mine = 0;
        const int keys = p.parts * p.top_k;
        const uint64_t* key = part_keys(p, (int64_t)row * p.parts);
        if (r.live) {
            if (r.target >= 0 && r.target < p.V) xt = D::load(x + r.target);
            if (lane < p.parts) {
                const float4 v = *part_sums(p, (int64_t)row * p.parts + lane);
                a = {v.x, v.y, v.z};
            }
            if (Top)
                for (int i = lane; i < keys; i += kThreads) mine = key[i] > mine ? key[i] : mine;
        }
        a = join_waves(a, scale2, shared);
        if (lane == 0) write_row(p, row, r, a, xt);
        if (Top) {
            const Scores c = scores_of(a);
            if (!r.live || c.m != c.m) {
                for (int k = lane; k < p.top_k; k += kThreads) write_top(p, row, k, 0, r.live, c);
            } else {
                sel.list[lane] = mine;
                __syncthreads();
                if (lane < 64) {
                    const uint64_t four[4] = {sel.list[lane], sel.list[lane + 64],
                                              sel.list[lane + 128], sel.list[lane + 192]};
                    const uint64_t from = kth_key(four, p.top_k);
                    if (lane == 0) {
                        sel.from = from;
                        sel.count = 0;
                    }
                }
                __syncthreads();
                const uint64_t from = sel.from;
                // (at most kMaxTop lanes reach it, with kMaxParts * kMaxTop / kThreads keys each)
                if (mine >= from)
                    for (int i = lane; i < keys; i += kThreads)
                        if (key[i] != 0 && key[i] >= from) push(sel, key[i]);
                __syncthreads();
                const int count = sel.count;
                for (int i = lane; i < count; i += kThreads) {
                    const uint64_t k = sel.list[i];
                    int rank = 0;
                    for (int j = 0; j < count; ++j) rank += sel.list[j] > k;
                    if (rank < p.top_k) write_top(p, row, rank, k, true, c);
                }
            }
        }
        __syncthreads();
    }
}

// ---- backward kernel

// 1 - e^l for l <= 0, without cancellation: its Taylor series where the ninth term is below 2^-31
// of the first.
__device__ __forceinline__ float one_minus_exp(float l, float e)
{
    if (l < -0.35f) return 1.f - e;
    float v = 1.f / 40320.f;
    v = v * l + 1.f / 5040.f;
    v = v * l + 1.f / 720.f;
    v = v * l + 1.f / 120.f;
    v = v * l + 1.f / 24.f;
    v = v * l + 1.f / 6.f;
    v = v * l + 0.5f;
    v = v * l + 1.f;
    return -v * l;
}

// What the gradient of a row takes, in units of log2: l2 = (x - m) * scale2 - logs2 is a logit's log2 p,
// and its gradient -2^l2 (c + h2 l2), the target's larger by g.
struct RowGrad {
    bool zero;
    float m, logs2, scale2, c, h2, g;
    int target;
};

template <bool Ent>
__device__ __forceinline__ RowGrad row_grad(const TokenGradParams& p, const SeqLengths& lens, uint32_t row)
{
    const Row r = row_of(p, lens, row / p.T, row % p.T);
    RowGrad w;
    const float logs = p.stats[2 * (int64_t)row + 1];
    w.m = p.stats[2 * (int64_t)row];
    w.zero = !r.live || !(w.m > -INFINITY) || r.target >= p.V;
    w.logs2 = logs * kLog2e;
    w.scale2 = p.scale * kLog2e;
    w.g = p.grad_logp ? p.grad_logp[row] * p.scale : 0.f;
    const float h = Ent ? p.grad_entropy[row] * p.scale : 0.f;
    w.c = Ent ? w.g + h * p.entropy[row] : w.g;
    w.h2 = h * kLn2;
    w.target = w.zero ? -1 : (int)r.target;
    return w;
}

template <bool Ent>
__device__ __forceinline__ float grad_of(const RowGrad& w, float x, bool target)
{
    float l2 = (x - w.m) * w.scale2 - w.logs2;
    if (Ent) l2 = fmaxf(l2, -1e4f);  // (of a masked logit 0 * -inf would be left)
    const float pr = exp2_of(l2);
    if (__builtin_expect(target, 0)) {  // 1 - p without cancellation where p is near 1
        l2 = fmaxf(l2, -1e4f);
        return w.g * one_minus_exp(l2 * kLn2, pr) - pr * (w.c - w.g + w.h2 * l2);
    }
    return Ent ? -pr * (w.c + w.h2 * l2) : -pr * w.c;
}

// G lanes a stretch of a row; p.pieces stretches of p.piece logits a row. Rows of up to that many
// logits are one stretch.
template <typename D, int G, bool Ent>
__global__ __launch_bounds__(kThreads) void k_token_grad(TokenGradParams p, SeqLengths lens)
{
    using Store = typename D::Store;
    constexpr int kRows = kThreads / G;
    const int lane = threadIdx.x % G;
    const uint64_t units = (uint64_t)p.B * p.T * p.pieces;
    for (uint64_t unit = (uint64_t)blockIdx.x * kRows + threadIdx.x / G; unit < units;
         unit += (uint64_t)gridDim.x * kRows) {
        const uint32_t row = p.pieces == 1 ? (uint32_t)unit : (uint32_t)(unit / p.pieces);
        const int from = p.pieces == 1 ? 0 : (int)(unit % p.pieces) * p.piece;
        const int n = p.V - from < p.piece ? p.V - from : p.piece;
        const int full = n / D::kVec;
        const RowGrad w = row_grad<Ent>(p, lens, row);
        const Store* x = static_cast<const Store*>(row_at(p, row / p.T, row % p.T, sizeof(Store))) + from;
        Store* out = static_cast<Store*>(p.grad) + (int64_t)row * p.V + from;
        if (w.zero) {
            for (int q = lane; q < full; q += G) store16(out + (int64_t)q * D::kVec, make_uint4(0, 0, 0, 0));
            for (int i = full * D::kVec + lane; i < n; i += G) D::store(out + i, 0.f);
            continue;
        }
        // (read before this group of lanes writes anything: the gradient may replace the logits)
        const int target = w.target - from;
        const float xt = w.target >= from && target < n ? D::load(x + target) : 0.f;
        for (int q = lane; q - lane < full; q += kLoads * G) {
            uint4 r[kLoads];
            load_group<D, G>(x, full, q, r);
#pragma unroll
            for (int k = 0; k < kLoads; ++k) {
                const int at = (q + k * G) * D::kVec;
                if (q + k * G >= full) break;
                float f[D::kVec];
                D::unpack(r[k], f);
#pragma unroll
                for (int i = 0; i < D::kVec; ++i) f[i] = grad_of<Ent>(w, f[i], false);
                store16(out + at, D::pack(f));
                if (__builtin_expect((uint32_t)(target - at) < (uint32_t)D::kVec, 0))
                    D::store(out + target, grad_of<Ent>(w, xt, true));
            }
        }
        for (int i = full * D::kVec + lane; i < n; i += G)
            D::store(out + i, grad_of<Ent>(w, D::load(x + i), i == target));
    }
}

}  // namespace

namespace {

template <typename D, bool Ent, bool Top>
void launch_rows(const TokenParams& p, const SeqLengths& lens, hipStream_t stream)
{
    const int64_t rows = (int64_t)p.B * p.T;
    const auto blocks = [](int64_t n) { return dim3((unsigned)(n < (1 << 20) ? n : 1 << 20)); };
    if (p.parts > 1) {
        k_token_blocks<D, Ent, Top, true><<<blocks(rows * p.parts), kThreads, 0, stream>>>(p, lens);
        k_token_join<D, Top><<<blocks(rows), kThreads, 0, stream>>>(p, lens);
    } else if (p.V > 4096) {
        k_token_blocks<D, Ent, Top, false><<<blocks(rows), kThreads, 0, stream>>>(p, lens);
    } else if (Top || p.V > 128) {
        k_token_rows<D, 64, Ent, Top><<<blocks((rows + 3) / 4), kThreads, 0, stream>>>(p, lens);
    } else {
        k_token_rows<D, 16, Ent, false><<<blocks((rows + 15) / 16), kThreads, 0, stream>>>(p, lens);
    }
}

template <typename D>
hipError_t launch_type(const TokenParams& p, const SeqLengths& lens, hipStream_t stream)
{
    if (p.entropy && p.top_k) launch_rows<D, true, true>(p, lens, stream);
    else if (p.entropy) launch_rows<D, true, false>(p, lens, stream);
    else if (p.top_k) launch_rows<D, false, true>(p, lens, stream);
    else launch_rows<D, false, false>(p, lens, stream);
    return hipGetLastError();
}

}  // namespace

TokenPlan plan_tokens(int64_t rows, int V, int top_k)
{
    TokenPlan plan{1, V, 0};
    // 1,024 workgroups fill the chip, and a part of 4,096 logits is worth a workgroup
    if (rows < 512 && V >= 8192) {
        int64_t parts = 1024 / rows;
        parts = parts < V / 4096 ? parts : V / 4096;
        parts = parts < kMaxParts ? parts : kMaxParts;
        if (parts > 1) {
            // (a multiple of 64 logits: parts of an aligned row are aligned)
            plan.part_size = (int)(((V + parts - 1) / parts + 63) / 64 * 64);
            plan.parts = (V + plan.part_size - 1) / plan.part_size;
            plan.workspace = (size_t)rows * plan.parts * (sizeof(float4) + sizeof(uint64_t) * top_k);
        }
    }
    return plan;
}

hipError_t launch_token_logprobs(const TokenParams& p, const SeqLengths& lens, int dtype,
                                 hipStream_t stream)
{
    if (dtype == LFMMI_F32) return launch_type<F32>(p, lens, stream);
    if (dtype == LFMMI_BF16) return launch_type<Bf16>(p, lens, stream);
    return launch_type<F16>(p, lens, stream);
}

namespace {

template <typename D, bool Ent>
hipError_t launch_grad(TokenGradParams p, const SeqLengths& lens, hipStream_t stream)
{
    const int64_t rows = (int64_t)p.B * p.T;
    const auto blocks = [](int64_t n) { return dim3((unsigned)(n < (1 << 20) ? n : 1 << 20)); };
    p.piece = p.V;
    p.pieces = 1;
    if (p.V <= 256) {
        k_token_grad<D, 16, Ent><<<blocks((rows + 15) / 16), kThreads, 0, stream>>>(p, lens);
    } else if (p.V <= 8192) {
        k_token_grad<D, 64, Ent><<<blocks((rows + 3) / 4), kThreads, 0, stream>>>(p, lens);
    } else {
        p.piece = kThreads * kLoads * D::kVec;
        p.pieces = (p.V + p.piece - 1) / p.piece;
        k_token_grad<D, kThreads, Ent><<<blocks(rows * p.pieces), kThreads, 0, stream>>>(p, lens);
    }
    return hipGetLastError();
}

template <typename D>
hipError_t launch_grad_type(const TokenGradParams& p, const SeqLengths& lens, hipStream_t stream)
{
    return p.grad_entropy ? launch_grad<D, true>(p, lens, stream) : launch_grad<D, false>(p, lens, stream);
}

}  // namespace

hipError_t launch_token_grad(const TokenGradParams& p, const SeqLengths& lens, int dtype,
                             hipStream_t stream)
{
    if (dtype == LFMMI_F32) return launch_grad_type<F32>(p, lens, stream);
    if (dtype == LFMMI_BF16) return launch_grad_type<Bf16>(p, lens, stream);
    return launch_grad_type<F16>(p, lens, stream);
}

}  // namespace lfmmi
