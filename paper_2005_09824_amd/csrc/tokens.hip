// Log probabilities of given tokens, with entropy and the best alternatives of every row of
// logits, and their gradient. See include/lfmmi.h for the formulas.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/lfmmi.h"
#include "lanes.h"
#include "operators.h"
#include "vec16.h"

namespace lfmmi {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.693147180559945309f;
constexpr int kThreads = 256;
constexpr int kLoads = 4;  // 16-byte loads that a lane has in flight

constexpr int threads_of(int lanes) { return lanes > kThreads ? lanes : kThreads; }

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

// What is the same in every lane of a wave, held once.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint64_t uniform(uint64_t v)
{
    return (uint64_t)uniform((uint32_t)(v >> 32)) << 32 | uniform((uint32_t)v);
}
__device__ __forceinline__ float uniform(float v) { return __uint_as_float(uniform(__float_as_uint(v))); }

// ---- reductions over a wave; every lane has the result

__device__ __forceinline__ uint32_t all_bits(uint32_t v)  // of a wave, and-ed
{
#define LFMMI_ROR(n) __builtin_amdgcn_update_dpp(v, v, 0x120 + n, 0xf, 0xf, true)
    v &= LFMMI_ROR(8);
    v &= LFMMI_ROR(4);
    v &= LFMMI_ROR(2);
    v &= LFMMI_ROR(1);
#undef LFMMI_ROR
    return (uint32_t)__builtin_amdgcn_readlane(v, 0) & (uint32_t)__builtin_amdgcn_readlane(v, 16) &
           (uint32_t)__builtin_amdgcn_readlane(v, 32) & (uint32_t)__builtin_amdgcn_readlane(v, 48);
}
__device__ __forceinline__ uint64_t all_bits(uint64_t v)
{
    return (uint64_t)all_bits((uint32_t)(v >> 32)) << 32 | all_bits((uint32_t)v);
}
__device__ __forceinline__ uint32_t max_of_two(uint32_t v)  // lanes next to each other
{
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(v, v, 0xb1, 0xf, 0xf, true));
}
__device__ __forceinline__ uint32_t max_of_four(uint32_t v)
{
    v = max_of_two(v);
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(v, v, 0x4e, 0xf, 0xf, true));
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
__device__ __forceinline__ float finite(float y) { return fmaxf(y, -1e20f); }

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

// Values in an order of whole numbers (-0 and 0 are equal); no value is 0.
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t v) { return __uint_as_float(v >> 31 ? v & 0x7fffffffu : ~v); }

// A value and its index as one whole number: equal values by index, lowest first.
__device__ __forceinline__ uint64_t key_of(float x, int i) { return (uint64_t)ordered(x) << 32 | (uint32_t)~i; }

struct Row {
    bool live;
    int target;  // -1: none, V: one that is not below V
};

// G: the lanes that take the row together.
template <int G, typename P>
__device__ __forceinline__ Row row_of(const P& p, const SeqLengths& lens, uint32_t row)
{
    if (lens.n > 0 && (int)(row % p.T) >= lens.T[row / p.T]) return {false, -1};
    if (!p.targets) return {true, -1};
    int64_t target = p.target_bytes == 8 ? static_cast<const int64_t*>(p.targets)[row]
                                         : static_cast<const int32_t*>(p.targets)[row];
    if (G >= 64) target = (int64_t)uniform((uint64_t)target);
    return {target >= 0, target < 0 ? -1 : target < p.V ? (int)target : p.V};
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
    // (s is 1 or more but for rounding: no log probability is above 0, no entropy below)
    return flags ? Scores{bad, bad} : Scores{a.m, log2f(fmaxf(a.s, 1.f)) * kLn2};
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
        entropy = flags == 2 ? NAN : flags == 1 ? 0.f : c.logs - kLn2 * fminf(a.u / a.s, 0.f);
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
    if (p.top_id) p.top_id[at] = live && !(c.m != c.m) ? (int)~(uint32_t)key : -1;
    if (p.top_logp)
        p.top_logp[at] = !live ? 0.f : c.m == -INFINITY ? -INFINITY
                                                        : (value_of((uint32_t)(key >> 32)) - c.m) * p.scale - c.logs;
}

// ---- one pass over n logits by G lanes

// Chunks of 16 bytes go round the lanes; a lane takes a group of kLoads of them at a time.
// `first`: the largest value a lane met in whole chunks (-inf to begin with), `group` the first
// group that held it, `second` the largest of the other groups.
struct Best {
    float first, second;
    int group;
};

__device__ __forceinline__ void take(Best& best, float top, int group)
{
    if (top > best.first) best.group = group;
    best.second = __builtin_amdgcn_fmed3f(best.first, best.second, top);
    best.first = fmaxf(best.first, top);
}

// A row of 16-bit logits that starts at an odd multiple of 2 is read from its second logit on (16-byte loads
// at odd multiples of 2 take 20 % longer than at 4): `head` is 1 then, and logit -1 comes with those behind
// the last whole chunk. The i-th of these:
__device__ __forceinline__ int single(int i, int behind, int head) { return i < head ? -1 : behind + i - head; }

template <typename D, int G>
__device__ __forceinline__ void load_part(const typename D::Store* x, int full, int q, uint4* r)
{
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        r[k] = make_uint4(D::kNone, D::kNone, D::kNone, D::kNone);
        if (q + k * G < full) r[k] = load16(x + (int64_t)(q + k * G) * D::kVec);
    }
}

template <int N>
__device__ __forceinline__ float max_of(const float (&f)[N])
{
    float top = f[0];
#pragma unroll
    for (int i = 1; i + 1 < N; i += 2) top = max3(top, f[i], f[i + 1]);
    return N % 2 ? top : fmaxf(top, f[N - 1]);
}

// Adds the first `chunks` chunks of a lane's logits, of any kind; a.m is their largest at least.
template <int N>
__device__ __forceinline__ void add_any(Sums& a, const float (&f)[N], int chunks, float scale2)
{
    constexpr int kVec = N < kLoads ? N : N / kLoads;
    float s[4] = {a.s, 0.f, 0.f, 0.f}, u[4] = {a.u, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i % kVec == 0 && i / kVec >= chunks) break;
        const float y = (f[i] - a.m) * scale2, e = exp2_of(y);
        s[i & 3] += e;
        u[i & 3] += e * finite(y);
    }
    a.s = (s[0] + s[1]) + (s[2] + s[3]);
    a.u = (u[0] + u[1]) + (u[2] + u[3]);
}

// The same with two operations less for each: y = x scale2 - c, c = m scale2 rounded, in one, and no
// clamp. What c is off by is taken out of the sums, to first order: not for |c| from 4,096 on (there
// `off` reaches 2^-12, and its square 2^-24). False, with nothing added, where 0 * -inf has come into u.
template <int N>
__device__ __forceinline__ bool add_plain(Sums& a, const float (&f)[N], float scale2)
{
    const float c = a.m * scale2, off = fmaf(a.m, scale2, -c);
    float s[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float y = fmaf(f[i], scale2, -c), e = exp2_of(y);
        s[i & 3] += e;
        u[i & 3] = fmaf(e, y, u[i & 3]);
    }
    float sum = (s[0] + s[1]) + (s[2] + s[3]);
    const float usum = (u[0] + u[1]) + (u[2] + u[3]);
    asm volatile("" : "+v"(sum));  // (added up here: after the branch all 2^y would be held until then)
    if (__builtin_amdgcn_ballot_w64(usum != usum)) return false;
    const float back = 1.f - off * kLn2;  // 2^-off
    a.s = fmaf(sum, back, a.s);
    a.u = fmaf(usum - off * sum, back, a.u);
    return true;
}

// Per logit of 16 bits: half an instruction for the maximum, one to unpack it, one for y, four
// issue slots for 2^y, one for each sum. `once`: the loads leave nothing in the caches.
template <typename D, int G, bool Top>
__device__ __forceinline__ void scan(const typename D::Store* x, int n, int head, int lane, float scale2, bool once,
                                     Sums& a, Best& best)
{
    constexpr int kVec = D::kVec, N = kVec * kLoads;
    const int full = n / kVec;
    bool plain = G > 16;  // until logits are met that add_plain does not take
    for (int q = lane, j = 0; q - lane < full; q += kLoads * G, ++j) {
        const int chunks = (full - (q - lane) + G - 1) / G;  // (the last group may have fewer)
        uint4 r[kLoads];
        if (G > 16 && q - lane + kLoads * G <= full) {
            if (once) {
#pragma unroll
                for (int k = 0; k < kLoads; ++k) r[k] = load16_once(x + (int64_t)(q + k * G) * kVec);
            } else {
#pragma unroll
                for (int k = 0; k < kLoads; ++k) r[k] = load16(x + (int64_t)(q + k * G) * kVec);
            }
        } else {
            load_part<D, G>(x, full, q, r);
            plain = false;
        }
        float f[N];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) D::unpack(r[k], f + k * kVec);
        const float top = max_of(f);
        if (Top) take(best, top, j);
        shift(a, fmaxf(a.m, top), scale2);
        plain = plain && !__builtin_amdgcn_ballot_w64(!(fabsf(a.m * scale2) < 4096.f));
        if (plain) plain = add_plain(a, f, scale2);
        if (!plain) add_any(a, f, chunks, scale2);
    }
    for (int i = lane; i < n - full * kVec + head; i += G) {
        const float f[1] = {D::load(x + single(i, full * kVec, head))};
        shift(a, fmaxf(a.m, f[0]), scale2);
        add_any(a, f, 1, scale2);
    }
}

// ---- the best alternatives
//
// The k-th largest, T, of the lanes' own largest values is a lower bound of the k-th largest
// value of the row, and rarely many more than k values reach it. They lie with the lanes whose
// largest does, in the group of chunks that the lane has noted, and anywhere with a lane whose second
// group does too: so one pass finds T, and few chunks are looked at again. What reaches T is put in
// order by counting, for each, how many are larger. Where more than kTies lanes over k reach T (equal
// logits) or T is -inf (masked rows) T gets an index as well, and where more values reach it than the list
// holds those in the list give a higher T.
constexpr int kTies = 32;
// Where k is kFew at most, 64 lanes' worth of maxima give a T that hardly more than k values reach; and T
// need not be the k-th exactly, the last few bits of it are left out.
constexpr int kFew = 32, kNear = 3;

// Of the N values that each lane of a wave holds, how many are from `c` on.
template <typename V, int N>
__device__ __forceinline__ int count_from(const V (&v)[N], V c)
{
    int count = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) count += __builtin_popcountll(__builtin_amdgcn_ballot_w64(v[i] >= c));
    return count;
}

// The k-th largest of them, or a lower bound of it with at most k + more values from there on; 0 if
// fewer than k are not 0. Bit by bit from the highest, bits in which no two values differ left out.
template <typename V, int N>
__device__ __forceinline__ V kth_value(const V (&v)[N], int k, int more)
{
    V all = v[0], none = ~v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) {
        all &= v[i];
        none &= ~v[i];
    }
    V t = all_bits(all), open = ~(t | all_bits(none));
    if (t == 0 && count_from(v, (V)1) < k) return 0;
    for (int count = 64 * N; open && count > k + more;) {
        const V bit = (V)1 << (63 - __builtin_clzll(open));
        const int above = count_from(v, (V)(t | bit));
        open ^= bit;
        if (above >= k) {
            t |= bit;
            count = above;
        }
    }
    return t;
}

// LDS of one row's selection.
template <int G>
struct Selection {
    static constexpr int kCap = G == 64 ? 512 : 1024;  // keys that it holds
    uint64_t list[kCap];
    uint32_t bins[G == 64 ? 1 : 256];
    int count;
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

// A value for each lane, to be read as each wave's share of all: with more than 256 lanes the
// largest of two or four.
template <int G>
__device__ __forceinline__ void put_bin(Selection<G>& sel, int lane, uint32_t v)
{
    if (G == 256) {
        sel.bins[lane] = v;
    } else if (G == 512) {
        v = max_of_two(v);
        if (lane % 2 == 0) sel.bins[lane / 2] = v;
    } else if (G == 1024) {
        v = max_of_four(v);
        if (lane % 4 == 0) sel.bins[lane / 4] = v;
    }
}
template <int G, int N>
__device__ __forceinline__ void get_bins(const Selection<G>& sel, int lane, uint32_t own, uint32_t (&v)[N])
{
    if (G == 64) {
        v[0] = own;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = sel.bins[lane % 64 + 64 * i];
    }
}

template <int G>
__device__ __forceinline__ void push(Selection<G>& sel, uint64_t key)
{
    const int at = atomicAdd(&sel.count, 1);
    if (at < Selection<G>::kCap) sel.list[at] = key;
}

// What the search for the values that reach (T, `last`) takes: larger ones, and equal ones
// of an index up to `last`. Indices count from the first of the n logits, keys from `offset`.
struct Bound {
    uint32_t value;
    int last, offset;
};

template <int G>
__device__ __forceinline__ void push_if(float v, int at, const Bound& to, Selection<G>& sel)
{
    const uint32_t o = ordered(v);
    if (o > to.value || (o == to.value && at <= to.last)) push(sel, (uint64_t)o << 32 | (uint32_t)~(to.offset + at));
}

template <int G>
__device__ __forceinline__ bool full_list(const Selection<G>& sel)
{
    return (int)uniform((uint32_t)*(volatile const int*)&sel.count) > Selection<G>::kCap;
}

// Each wave looks through what its own lanes have read, a chunk a lane.
template <typename D, int G>
__device__ __forceinline__ void gather(const typename D::Store* x, int n, int head, int lane, const Best& best,
                                       const Bound& to, Selection<G>& sel)
{
    constexpr int kVec = D::kVec;
    const int full = n / kVec, in_wave = lane % 64, base = lane - in_wave;
    const uint32_t first = ordered(best.first), second = ordered(best.second);
    const int start = (best.group * kLoads * G + lane) * kVec;  // the lowest index it can have
    const bool in = lane < full && (first > to.value || (first == to.value && start <= to.last) || to.value == 0);
    // (if both are equal to T the second one's group comes later)
    const bool later = first == to.value && (best.group + 1) * kLoads * G * kVec > to.last;
    const bool deep = in && (second > to.value || (second == to.value && !later) || to.value == 0);
    const uint64_t ones = __builtin_amdgcn_ballot_w64(in && !deep), deeps = __builtin_amdgcn_ballot_w64(deep);
    const int num_one = __builtin_popcountll(ones), num_deep = __builtin_popcountll(deeps);
    if (num_one + num_deep > 0) {
        // lanes of one group, then lanes of all groups, then the others, in a row
        const uint64_t below = ((uint64_t)1 << in_wave) - 1;
        const int one = __builtin_popcountll(ones & below), far = __builtin_popcountll(deeps & below);
        const int slot = deep ? num_one + far : in ? one : num_one + num_deep + in_wave - one - far;
        const int sent = __builtin_amdgcn_ds_permute(slot * 4, best.group << 6 | in_wave);
        const int each = (full + G - 1) / G;  // chunks of a lane, at most
        const int items = num_one * kLoads + num_deep * each;
        const float least = value_of(max(to.value, ordered(-INFINITY)));  // (below that bits are no number's)
        // (a list that is full is only there to give a better bound)
        for (int w = in_wave; w - in_wave < items && !full_list(sel); w += 64) {
            const int all = w - num_one * kLoads;
            const int from = all < 0 ? w / kLoads : num_one + all / each;
            const int v = __builtin_amdgcn_ds_bpermute((from & 63) * 4, sent);
            const int q = (all < 0 ? (v >> 6) * kLoads + w % kLoads : all % each) * G + base + (v & 63);
            if (w < items && q < full) {
                float f[kVec];
                D::unpack(load16(x + (int64_t)q * kVec), f);
                uint32_t hits = 0;
#pragma unroll
                for (int i = 0; i < kVec; ++i) hits |= f[i] >= least ? 1u << i : 0u;
                for (; hits; hits &= hits - 1) {  // (few: the value is loaded once more)
                    const int at = q * kVec + __builtin_ctz(hits);
                    push_if<G>(D::load(x + at), at, to, sel);
                }
            }
        }
    }
    for (int i = lane; i < n - full * kVec + head; i += G) {
        const int at = single(i, full * kVec, head);
        push_if<G>(D::load(x + at), at, to, sel);
    }
}

// The index that goes with T: k lanes hold a larger value, or T at an index up to it.
template <typename D, int G, int N>
__device__ __forceinline__ int last_index(const typename D::Store* x, int n, int lane, const Best& best,
                                          uint32_t value, int k, const uint32_t (&v)[N], Selection<G>& sel)
{
    const int full = n / D::kVec, larger = count_from(v, value + 1);
    if (larger >= k) return INT32_MAX;  // (a bound that no lane's value is equal to)
    uint32_t mine = 0;
    if (lane < full && ordered(best.first) == value) {
        int at = 0;
#pragma unroll
        for (int i = kLoads - 1; i >= 0; --i) {
            const int q = (best.group * kLoads + i) * G + lane;
            if (q >= full) continue;
            float f[D::kVec];
            D::unpack(load16(x + (int64_t)q * D::kVec), f);
#pragma unroll
            for (int e = D::kVec - 1; e >= 0; --e)
                if (f[e] == best.first) at = q * D::kVec + e;
        }
        mine = ~(uint32_t)at;
    }
    uint32_t w[N];
    row_sync<G>();
    put_bin(sel, lane, mine);
    row_sync<G>();
    get_bins(sel, lane, mine, w);
    return (int)~kth_value(w, k - larger, 0);
}

// A bound of the list's k-th largest key, from every wave's own look at it.
template <int G>
__device__ __forceinline__ uint64_t bound_of_list(int lane, int k, int count, const Selection<G>& sel)
{
    uint64_t v[Selection<G>::kCap / 64];
#pragma unroll
    for (int i = 0; i < Selection<G>::kCap / 64; ++i)
        v[i] = lane % 64 + 64 * i < count ? sel.list[lane % 64 + 64 * i] : 0;
    return kth_value(v, k, kNear);
}

// Leaves of a list of many keys those that can be among the k largest. Returns their number.
constexpr int kMany = 192;
template <int G>
__device__ __forceinline__ int thin_out(int lane, int k, int count, Selection<G>& sel)
{
    constexpr int kEach = Selection<G>::kCap / G;
    const uint64_t from = bound_of_list(lane, k, count, sel);
    uint64_t mine[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) mine[j] = lane + j * G < count ? sel.list[lane + j * G] : 0;
    row_sync<G>();
    if (lane == 0) sel.count = 0;
    row_sync<G>();
#pragma unroll
    for (int j = 0; j < kEach; ++j)
        if (mine[j] && mine[j] >= from) push(sel, mine[j]);
    row_sync<G>();
    return sel.count;
}

template <int G, typename Put>
__device__ __forceinline__ void put_ranked(int lane, int k, int count, const Selection<G>& sel, Put&& put)
{
    for (int i = lane; i < count; i += G) {
        const uint64_t key = sel.list[i];
        int rank = 0;
        for (int j = 0; j < count; j += 8) {  // (the list has a multiple of 8 places)
            uint64_t other[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) other[e] = sel.list[j + e];
#pragma unroll
            for (int e = 0; e < 8; ++e) rank += j + e < count && other[e] > key;
        }
        if (rank < k) put(rank, key);
    }
}

// Before the sync that select_top is called behind.
template <typename D, int G>
__device__ __forceinline__ uint32_t offer(int n, int lane, const Best& best, Selection<G>& sel)
{
    const uint32_t own = lane < n / D::kVec ? ordered(best.first) : 0;
    put_bin(sel, lane, own);
    if (lane == 0) sel.count = 0;
    return own;
}

// The k best of n logits, handed to put(rank, key) by the lane that has one. `own`: what offer gave.
template <typename D, int G, typename Put>
__device__ __forceinline__ void select_top(const typename D::Store* x, int n, int head, int lane, int offset, int k,
                                           const Best& best, uint32_t own, Selection<G>& sel, Put&& put)
{
    constexpr int kCap = Selection<G>::kCap;
    uint32_t v[G == 64 ? 1 : 4];
    get_bins(sel, lane, own, v);
    Bound to{0, INT32_MAX, offset};
    if (G > 64 && k <= kFew) {
        const uint32_t most[1] = {max(max(v[0], v[G > 64 ? 1 : 0]), max(v[G > 64 ? 2 : 0], v[G > 64 ? 3 : 0]))};
        to.value = kth_value(most, k, kNear);
    } else {
        to.value = kth_value(v, k, kNear);
    }
    if (to.value && (to.value == ordered(-INFINITY) || count_from(v, to.value) > k + kTies))
        to.last = last_index<D, G>(x, n, lane, best, to.value, k, v, sel);
    gather<D, G>(x, n, head, lane, best, to, sel);
    row_sync<G>();
    int count = sel.count;
    while (__builtin_expect(count > kCap, 0)) {
        // What the list holds gives a higher bound, which at least kCap - k - kNear keys fewer reach.
        const uint64_t from = bound_of_list(lane, k, kCap, sel);
        to.value = (uint32_t)(from >> 32);
        to.last = (int)min(~(uint32_t)from, (uint32_t)INT32_MAX) - offset;
        row_sync<G>();
        if (lane == 0) sel.count = 0;
        row_sync<G>();
        gather<D, G>(x, n, head, lane, best, to, sel);
        row_sync<G>();
        count = sel.count;
    }
    if (count > kMany) count = thin_out(lane, k, count, sel);
    put_ranked(lane, k, count, sel, put);
}

// ---- forward kernels

template <typename P>
__device__ __forceinline__ const void* row_at(const P& p, uint32_t row, size_t size)
{
    return static_cast<const char*>(p.x) +
           ((int64_t)(row / p.T) * p.stride_b + (int64_t)(row % p.T) * p.stride_t) * (int64_t)size;
}

template <typename D, int G>
__device__ __forceinline__ float target_logit(const typename D::Store* x, const Row& r, int V)
{
    if (r.target < 0 || r.target >= V) return 0.f;
    const float v = D::load(x + r.target);
    return G >= 64 ? uniform(v) : v;
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

// The sums of G lanes; every lane has them. With more than a wave behind a sync.
template <int G>
__device__ __forceinline__ Sums join_all(Sums a, float scale2, Sums* shared)
{
    join_lanes<(G < 64 ? G : 64)>(a, scale2);
    if (G > 64) {
        if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64] = a;
        __syncthreads();
        // (each 16 lanes of a wave join what the waves have, at most 16, once more)
        a = threadIdx.x % 16 < G / 64 ? shared[threadIdx.x % 16] : no_sums();
        join_lanes<16>(a, scale2);
        a = {uniform(a.m), uniform(a.s), uniform(a.u)};
    }
    return a;
}

// G lanes a row, or for Split G lanes for each of p.parts parts of a row. Bound by the reads where rows are
// many: 6,144 rows of 65,536 bf16 132 us, 6.1 TB/s (16-byte loads alone reach 6.9); 2,570 of 131,072 with 5
// alternatives 116 us, 5.8 TB/s, of which the selection takes 6 us; by latency where they are few: one of 32,000
// with 8 alternatives 7.4 us, 4.4 without.
template <typename D, int G, bool Top, bool Split>
__global__ __launch_bounds__(threads_of(G)) void k_token(TokenParams p, SeqLengths lens)
{
    static_assert(!Top || G >= 64, "a selection takes a wave");
    using Store = typename D::Store;
    constexpr int kRows = threads_of(G) / G;
    __shared__ Sums shared[G > 64 ? G / 64 : 1];
    __shared__ Selection<(G < 64 ? 64 : G)> sels[Top ? kRows : 1];
    const int lane = threadIdx.x % G, sub = threadIdx.x / G;
    auto& sel = sels[Top ? sub : 0];
    const float scale2 = p.scale * kLog2e;
    // (rows are below 2^31, and those of several parts few: sums with a grid fit 32 bits)
    const uint32_t units = (uint32_t)p.B * p.T * (Split ? p.parts : 1);
    for (uint32_t at = blockIdx.x * kRows + sub; at < units; at += gridDim.x * kRows) {
        const uint32_t unit = G == 64 ? uniform(at) : at;
        const uint32_t row = Split ? unit / p.parts : unit;
        const int begin = Split ? (int)(unit % p.parts) * p.part_size : 0;
        const int all = Split ? (p.V - begin < p.part_size ? p.V - begin : p.part_size) : p.V;
        const Row r = row_of<G>(p, lens, row);
        const Store* x = static_cast<const Store*>(row_at(p, row, sizeof(Store))) + begin;
        if (!r.live) {
            if (Split) continue;
            if (lane == 0) write_row(p, row, r, no_sums(), 0.f);
            if (Top)
                for (int k = lane; k < p.top_k; k += G) write_top(p, row, k, 0, false, Scores{0.f, 0.f});
            continue;
        }
        Sums a = no_sums();
        Best best{-INFINITY, -INFINITY, 0};
        const float xt = Split ? 0.f : target_logit<D, G>(x, r, p.V);
        const int head = (uintptr_t)x % 4 ? 1 : 0, n = all - head;
        x += head;
        scan<D, G, Top>(x, n, head, lane, scale2, p.once, a, best);
        const uint32_t own = Top ? offer<D>(n, lane, best, sel) : 0;
        a = join_all<G>(a, scale2, shared);
        if (lane == 0) {
            if (Split) *part_sums(p, unit) = make_float4(a.m, a.s, a.u, 0.f);
            else write_row(p, row, r, a, xt);
        }
        if (Top) {
            const Scores c = scores_of(a);
            if (c.m != c.m || c.m == -INFINITY) {  // no alternatives, or the first tokens
                for (int k = lane; k < p.top_k; k += G) {
                    const uint64_t key = c.m != c.m || k >= all ? 0 : key_of(-INFINITY, begin + k);
                    if (Split) part_keys(p, unit)[k] = key;
                    else write_top(p, row, k, key, true, c);
                }
            } else {
                row_sync<(G < 64 ? 64 : G)>();
                const int k = p.top_k < all ? p.top_k : all;
                select_top<D>(x, n, head, lane, begin + head, k, best, own, sel, [&](int rank, uint64_t key) {
                    if (Split) part_keys(p, unit)[rank] = key;
                    else write_top(p, row, rank, key, true, c);
                });
                if (Split)
                    for (int rank = k + lane; rank < p.top_k; rank += G) part_keys(p, unit)[rank] = 0;
            }
        }
        if (G > 64) __syncthreads();
        else if (Top) row_sync<64>();
    }
}

// Rows of up to 64 kEach logits with alternatives, a wave a row: the logits stay in registers, and take the
// place of the lanes' maxima in the selection.
template <typename D, int kEach>
__global__ __launch_bounds__(kThreads) void k_token_short(TokenParams p, SeqLengths lens)
{
    using Store = typename D::Store;
    constexpr int kRows = kThreads / 64;
    __shared__ Selection<64> sels[kRows];
    const int lane = threadIdx.x % 64;
    auto& sel = sels[threadIdx.x / 64];
    const float scale2 = p.scale * kLog2e;
    const uint32_t rows = (uint32_t)p.B * p.T;
    for (uint32_t at = blockIdx.x * kRows + threadIdx.x / 64; at < rows; at += gridDim.x * kRows) {
        const uint32_t row = uniform(at);
        const Row r = row_of<64>(p, lens, row);
        const Store* x = static_cast<const Store*>(row_at(p, row, sizeof(Store)));
        if (!r.live) {
            if (lane == 0) write_row(p, row, r, no_sums(), 0.f);
            if (lane < p.top_k) write_top(p, row, lane, 0, false, Scores{0.f, 0.f});
            continue;
        }
        const float xt = target_logit<D, 64>(x, r, p.V);
        float f[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) f[i] = lane + 64 * i < p.V ? D::load(x + lane + 64 * i) : -INFINITY;
        if (lane == 0) sel.count = 0;
        Sums a = no_sums();
        a.m = max_over<64>(fmaxf(a.m, max_of(f)));
        add_any(a, f, kLoads, scale2);
        a.s = sum_over<64>(a.s);
        a.u = sum_over<64>(a.u);
        if (lane == 0) write_row(p, row, r, a, xt);
        const Scores c = scores_of(a);
        if (c.m != c.m) {
            if (lane < p.top_k) write_top(p, row, lane, 0, true, c);
            continue;
        }
        uint32_t v[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i] = lane + 64 * i < p.V ? ordered(f[i]) : 0;
        const uint32_t least = kth_value(v, p.top_k, kNear);
        uint32_t least_index = 0;  // ~index that the values equal to `least` have to reach
        if (count_from(v, least) > kMany) {  // equal logits
            const int larger = count_from(v, least + 1);
            uint32_t w[kEach];
#pragma unroll
            for (int i = 0; i < kEach; ++i) w[i] = v[i] == least ? ~(uint32_t)(lane + 64 * i) : 0;
            if (larger < p.top_k) least_index = kth_value(w, p.top_k - larger, kNear);
        }
        row_sync<64>();
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t index = ~(uint32_t)(lane + 64 * i);
            if (v[i] && (v[i] > least || (v[i] == least && index >= least_index)))
                push(sel, (uint64_t)v[i] << 32 | index);
        }
        row_sync<64>();
        put_ranked(lane, p.top_k, sel.count, sel,
                   [&](int rank, uint64_t key) { write_top(p, row, rank, key, true, c); });
        row_sync<64>();
    }
}

// A workgroup a row: joins the parts' sums and alternatives, of which a lane has one (a key of 0 stands for
// none, and at least top_k are others). 256 ranked at once took 4 us more than behind a bound; 128 take
// a few tenths less.
template <typename D, bool Top>
__global__ __launch_bounds__(kThreads) void k_token_join(TokenParams p, SeqLengths lens)
{
    using Store = typename D::Store;
    static_assert(kMaxPartKeys <= kThreads && kMaxParts <= kThreads, "a lane has one");
    constexpr int kAtOnce = 128;
    __shared__ Sums shared[kThreads / 64];
    __shared__ Selection<kThreads> sel;
    const int lane = threadIdx.x;
    const float scale2 = p.scale * kLog2e;
    const uint32_t rows = (uint32_t)p.B * p.T;
    for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const Row r = row_of<kThreads>(p, lens, row);
        const Store* x = static_cast<const Store*>(row_at(p, row, sizeof(Store)));
        Sums a = no_sums();
        const int keys = p.parts * p.top_k;
        uint64_t mine = 0;
        float xt = 0.f;
        if (r.live) {
            xt = target_logit<D, kThreads>(x, r, p.V);
            if (lane < p.parts) {
                const float4 v = *part_sums(p, (int64_t)row * p.parts + lane);
                a = {v.x, v.y, v.z};
            }
            if (Top) {
                if (lane < keys) mine = part_keys(p, (int64_t)row * p.parts)[lane];
                sel.list[lane] = mine;
                if (lane == 0) sel.count = 0;
            }
        }
        a = join_all<kThreads>(a, scale2, shared);
        if (lane == 0) write_row(p, row, r, a, xt);
        if (Top) {
            const Scores c = scores_of(a);
            if (!r.live || c.m != c.m) {
                for (int k = lane; k < p.top_k; k += kThreads) write_top(p, row, k, 0, r.live, c);
            } else {
                int count = keys;
                if (keys > kAtOnce) {
                    uint64_t v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = sel.list[lane % 64 + 64 * i];
                    const uint64_t bound = kth_value(v, p.top_k, 0);
                    __syncthreads();
                    if (mine >= bound) push(sel, mine);
                    __syncthreads();
                    count = sel.count;
                }
                put_ranked(lane, p.top_k, count, sel,
                           [&](int rank, uint64_t key) { write_top(p, row, rank, key, true, c); });
            }
        }
        __syncthreads();
    }
}

// ---- backward kernel

// 1 - e^l for l <= 0, good to a few roundings of itself: its Taylor series where the ninth term is below
// 2^-30 of the first.
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
// and its gradient -2^l2 (c + h2 l2), with c = g + hent; the target's is larger by g.
struct RowGrad {
    bool zero;
    float m, logs2, scale2, c, h2, g, hent;
    int target;
};

template <int G, bool Ent>
__device__ __forceinline__ RowGrad row_grad(const TokenGradParams& p, const SeqLengths& lens, uint32_t row)
{
    const Row r = row_of<G>(p, lens, row);
    RowGrad w;
    const float logs = p.stats[2 * (int64_t)row + 1];
    w.m = p.stats[2 * (int64_t)row];
    w.zero = !r.live || !(w.m > -INFINITY) || r.target >= p.V;
    w.logs2 = logs * kLog2e;
    w.scale2 = p.scale * kLog2e;
    w.g = p.grad_logp ? p.grad_logp[row] * p.scale : 0.f;
    const float h = Ent ? p.grad_entropy[row] * p.scale : 0.f;
    w.hent = Ent ? h * p.entropy[row] : 0.f;
    w.c = w.g + w.hent;
    w.h2 = h * kLn2;
    w.target = w.zero ? -1 : r.target;
    return w;
}

template <bool Ent>
__device__ __forceinline__ float grad_of(const RowGrad& w, float x, bool target)
{
    float l2 = (x - w.m) * w.scale2 - w.logs2;
    if (Ent) l2 = fmaxf(l2, -1e4f);  // (of a masked logit 0 * -inf would be left)
    const float pr = exp2_of(l2);
    if (__builtin_expect(target, 0)) {
        // Where p is near 1 both terms are small beside g: 1 - p comes from l, as good as ln s is (a sum of
        // 32 bits beside 1: log p is off by some 2^-24), and g is not added to the second only to be taken off
        // again (2 % of a gradient at p = 1 - 1e-5 were rounding then).
        l2 = fmaxf(l2, -1e4f);
        return w.g * one_minus_exp(l2 * kLn2, pr) - pr * (w.hent + w.h2 * l2);
    }
    return Ent ? -pr * (w.c + w.h2 * l2) : -pr * w.c;
}

// Bound by HBM: 6,144 rows of 65,536 bf16 read and 8,192 written 316 us, 6.0 TB/s (a copy reaches 5.7, here some
// comes from the cache).
// G lanes a stretch of a row; p.pieces stretches of p.piece logits a row. Rows of up to that many
// logits are one stretch.
template <typename D, int G, bool Ent>
__global__ __launch_bounds__(kThreads) void k_token_grad(TokenGradParams p, SeqLengths lens)
{
    using Store = typename D::Store;
    constexpr int kRows = kThreads / G;
    const int lane = threadIdx.x % G;
    const uint32_t rows = (uint32_t)p.B * p.T;
    const uint32_t at = kRows == 1 ? blockIdx.y : blockIdx.x * kRows + threadIdx.x / G;
    const uint32_t step = kRows == 1 ? gridDim.y : gridDim.x * kRows;
    // (with one row a workgroup its pieces are next to each other in the order of the grid: rows first
    // took 11 % longer on 8,192 rows of 65,536)
    for (uint32_t row = G == 64 ? uniform(at) : at; row < rows; row += step)
    for (int piece = kRows == 1 ? blockIdx.x : 0; piece < p.pieces; piece += kRows == 1 ? gridDim.x : 1) {
        const int from = piece * p.piece;
        const int n = p.V - from < p.piece ? p.V - from : p.piece;
        const int full = n / D::kVec;
        const RowGrad w = row_grad<G, Ent>(p, lens, row);
        const Store* x = static_cast<const Store*>(row_at(p, row, sizeof(Store))) + from;
        Store* out = static_cast<Store*>(p.grad) + (int64_t)row * p.V + from;
        if (w.zero) {
            for (int q = lane; q < full; q += G) {
                if (p.once) store16_once(out + (int64_t)q * D::kVec, make_uint4(0, 0, 0, 0));
                else store16(out + (int64_t)q * D::kVec, make_uint4(0, 0, 0, 0));
            }
            for (int i = full * D::kVec + lane; i < n; i += G) D::store(out + i, 0.f);
            continue;
        }
        // (read before this group of lanes writes anything: the gradient may replace the logits)
        const int target = w.target - from;
        const float xt = w.target >= from && target < n ? D::load(x + target) : 0.f;
        for (int q = lane; q - lane < full; q += kLoads * G) {
            uint4 r[kLoads];
            if (p.once && q - lane + kLoads * G <= full) {
#pragma unroll
                for (int k = 0; k < kLoads; ++k) r[k] = load16_once(x + (int64_t)(q + k * G) * D::kVec);
            } else {
                load_part<D, G>(x, full, q, r);
            }
#pragma unroll
            for (int k = 0; k < kLoads; ++k) {
                const int first = (q + k * G) * D::kVec;
                if (q + k * G >= full) break;
                float f[D::kVec];
                D::unpack(r[k], f);
#pragma unroll
                for (int i = 0; i < D::kVec; ++i) f[i] = grad_of<Ent>(w, f[i], false);
                if (p.once) store16_once(out + first, D::pack(f));
                else store16(out + first, D::pack(f));
                if (__builtin_expect((uint32_t)(target - first) < (uint32_t)D::kVec, 0))
                    D::store(out + target, grad_of<Ent>(w, xt, true));
            }
        }
        for (int i = full * D::kVec + lane; i < n; i += G)
            D::store(out + i, grad_of<Ent>(w, D::load(x + i), i == target));
    }
}

constexpr int kComputeUnits = 256, kManyRows = 2048;
constexpr int kRowOf16 = 512;                                                   // logits
constexpr int64_t kWaveRow = 32 << 10, kLongRow = 64 << 10;                       // bytes

template <typename D, bool Top>
void launch_rows(const TokenParams& p, const SeqLengths& lens, hipStream_t stream)
{
    const int64_t rows = (int64_t)p.B * p.T;
    const auto blocks = [](int64_t n) { return dim3((unsigned)(n < (1 << 20) ? n : 1 << 20)); };
    const int64_t bytes = (int64_t)p.V * sizeof(typename D::Store);
    // Lanes a row. Microseconds a call in a replayed graph, the same rows each time (the caches hold them), bf16,
    // without / with 8 alternatives, at 64, 256, 1,024 lanes:
    //   4,096 rows of 12,000: 18.1 / 21.1, 21.1 / 31.0; 4,096 of 16,384: 23.8 / 27.5, 23.0 / 32.9;
    //   64 of 8,192: 4.8 / 7.6, 3.5 / 5.9; 256 of 8,192: -, 3.6 / 5.9, 4.3 / 7.5;
    //   256 of 65,536: -, 8.9 / 11.5, 7.0 / 10.3 (a compute unit holds one workgroup of 1,024, two of 512);
    // at 256, 512 and 1,024 lanes: 64 of 8,192: 3.5 / 5.9, 3.6 / 6.3, -; 64 of 16,384: 4.1 / 6.6, 3.8 / 6.5,
    //   4.1 / 7.6; 64 of 32,000: 5.6 / 8.2, 4.9 / 7.6, 4.7 / 8.3; 64 of 65,536: -, 6.8 / 9.5, 6.2 / 9.7; 128 of
    //   200,000, with 64 alternatives: -, 16.8 / 23.5, 15.3 / 21.6;
    // of more rows than compute units at 256 and 512 lanes: 257 of 32,000: 6.5 / 9.2, 6.4 / 9.9; 257 of 65,536:
    //   11.3 / 14.1, 10.0 / 13.3, with 64 alternatives 17.5, 15.6; 512 of 65,536: 13.1 / 16.0, 13.4 / 16.7,
    //   with 64 20.1, 18.4; 768: 18.9 / 21.8, 19.0 / 23.6, with 64 25.8, 27.9.
    // 32,000 rows without alternatives at 16 and 64 lanes: 84 logits 5.4, 15.1; 512: 7.5, 14.8 (fp32
    // 12.0, 13.9). Alternatives from registers and from lanes' maxima: 40,000 rows of 84, 8 of them, 33, 61;
    // 20,000 of 500, 5 of them, 34, 28, 64 of them 50, 78.
    // Other rows each time take 0.3 to 4 us more on both sides; the order turns only where these are less than 1 us
    // apart (512 and 768 of 65,536 without alternatives: 16.2, 15.3 and 22.8, 22.1).
    if (p.parts > 1) {
        k_token<D, 256, Top, true><<<blocks(rows * p.parts), 256, 0, stream>>>(p, lens);
        k_token_join<D, Top><<<blocks(rows), kThreads, 0, stream>>>(p, lens);
    } else if (bytes >= (Top ? 3 : 1) * kLongRow && rows <= kComputeUnits) {
        k_token<D, 1024, Top, false><<<blocks(rows), 1024, 0, stream>>>(p, lens);
    } else if (rows <= kComputeUnits
                   ? bytes >= kLongRow / 2
                   : bytes >= kLongRow && rows <= (p.top_k > kFew ? 2 * kComputeUnits : 3 * kComputeUnits / 2)) {
        k_token<D, 512, Top, false><<<blocks(rows), 512, 0, stream>>>(p, lens);
    } else if (bytes > (rows < kManyRows || p.top_k > kFew ? kWaveRow / 4 : kWaveRow)) {
        k_token<D, 256, Top, false><<<blocks(rows), 256, 0, stream>>>(p, lens);
    } else if (Top && p.V <= 128) {
        k_token_short<D, 2><<<blocks((rows + 3) / 4), kThreads, 0, stream>>>(p, lens);
    } else if (Top && p.V <= 256) {
        k_token_short<D, 4><<<blocks((rows + 3) / 4), kThreads, 0, stream>>>(p, lens);
    } else if (p.top_k > kFew && p.V <= 512) {
        k_token_short<D, 8><<<blocks((rows + 3) / 4), kThreads, 0, stream>>>(p, lens);
    } else if (Top || p.V > kRowOf16) {
        k_token<D, 64, Top, false><<<blocks((rows + 3) / 4), kThreads, 0, stream>>>(p, lens);
    } else {
        k_token<D, 16, false, false><<<blocks((rows + 15) / 16), kThreads, 0, stream>>>(p, lens);
    }
}

template <typename D>
hipError_t launch_type(const TokenParams& p, const SeqLengths& lens, hipStream_t stream)
{
    if (p.top_k) launch_rows<D, true>(p, lens, stream);
    else launch_rows<D, false>(p, lens, stream);
    return hipGetLastError();
}

}  // namespace

TokenPlan plan_tokens(int64_t rows, int V, int top_k)
{
    TokenPlan plan{1, V, 0};
    // A compute unit alone takes 0.05 us for 1,000 logits; in parts there is a second launch, and a second
    // selection that grows with the alternatives. Microseconds whole and in parts, without / with 8 alternatives,
    // the same rows each time, bf16: 1 of 131,072: 8.9 / 12.4, 5.2 / 9.2; 32: 9.3 / 12.9, 6.1 / 12.1; 64 of
    // 160,000: 11.7 / 15.4, 8.8 / 13.5; 64 of 100,000: 8.6 / 12.3, 7.2 / 11.9; with 20, 48 of 131,072: 13.6, 14.2;
    // with 64, 16 of 131,072: 15.3, 16.4, of 200,000: 19.7, 18.7; fp32 without, 33 of 50,021: 5.9, 6.0.
    // Other rows each time take 0.3 to 4 us more on both sides; the order turns only where these are less than 1 us
    // apart (with 64, 16 of 200,000: 21.8, 22.5; with 20, 48 of 128,000 fp16, 14.7, 14.9 else: 16.5, 16.3).
    const int64_t least = 65536 + (top_k ? 16384 + 768 * rows + 1024 * top_k : 512 * rows);
    if (rows <= 64 && V >= least) {
        // Two workgroups a compute unit, a part of 4,096 logits is worth one, and a lane of the join an
        // alternative: 64 of them for each of 24 parts took 25 us, of 4 parts 16.5.
        const int64_t parts = std::min<int64_t>(
            {2 * kComputeUnits / rows, V / 4096, kMaxParts, top_k ? kMaxPartKeys / top_k : kMaxParts});
        // (a multiple of 64 logits: parts of an aligned row are aligned)
        plan.part_size = (int)(((V + parts - 1) / parts + 63) / 64 * 64);
        plan.parts = (V + plan.part_size - 1) / plan.part_size;
        plan.workspace = (size_t)rows * plan.parts * (sizeof(float4) + sizeof(uint64_t) * top_k);
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
        // (a launch has fewer than 2^32 threads)
        const int64_t x = p.pieces < (1 << 20) ? p.pieces : 1 << 20, most = (1 << 22) / x;
        const int64_t y = rows < 65535 ? rows : 65535;
        const dim3 grid((unsigned)x, (unsigned)(y < most ? y : most));
        k_token_grad<D, kThreads, Ent><<<grid, kThreads, 0, stream>>>(p, lens);
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
