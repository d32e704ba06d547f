// Drafted tokens against the logits of the model that they are drafted for. See include/lfmmi.h for the rule.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/lfmmi.h"
#include "lanes.h"
#include "layers.h"
#include "rows.h"
#include "vec16.h"

namespace lfmmi {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kChunks = kVerifyPart / 8 / 64;  // of eight logits, that a lane takes of a part: a part is a wave's
constexpr int kRestThreads = 256;
constexpr int kRestParts = kRestThreads / 128;  // two waves a part
constexpr int kPickThreads = 512;

// What a part of a row comes to: its largest logit m, the sum s of exp(scale (x - m)) (0 of nothing but -inf, NaN where a logit
// is NaN or +inf), the first index of the largest.
struct Part {
    double s;
    float m;
    int first;
};

enum Kind { kLost, kAll, kDrafted, kGiven };  // what the last token is drawn from: nothing, p, p - q, p without the drafted one
struct Choice {  // the row that ends a sequence, its flags, a token (greedy: the best; kGiven: the drafted one)
    int row, flags, kind, token;
    float m, mq;      // largest logits of the target's row and the draft's
    double per, per_q;  // 1 / sums of those rows
};

struct Space {  // of the workspace
    Part* parts;      // [B, 2 K + 1, parts]: K + 1 rows of the target, K of the draft
    Choice* choice;   // [B]
    double* rest;     // [B, parts]: sums of what is left of p - q
};
__host__ __device__ size_t up(size_t bytes) { return (bytes + 15) / 16 * 16; }
__host__ __device__ size_t space_of(void* workspace, int64_t B, int K, int parts, Space* s)
{
    char* at = static_cast<char*>(workspace);
    const size_t rows = up((size_t)B * (2 * (size_t)K + 1) * parts * sizeof(Part)), choices = up((size_t)B * sizeof(Choice));
    if (s) {
        s->parts = reinterpret_cast<Part*>(at);
        s->choice = reinterpret_cast<Choice*>(at + rows);
        s->rest = reinterpret_cast<double*>(at + rows + choices);
    }
    return rows + choices + up((size_t)B * parts * sizeof(double));
}

__device__ __forceinline__ int drafts_of(const VerifyParams& p, const SeqLengths& lens, int b)
{
    return lens.n == 0 ? p.K : lens.T[b];
}
__device__ __forceinline__ int64_t drafted(const VerifyParams& p, int b, int i)
{
    const int64_t at = (int64_t)b * p.K + i;
    return p.token_bytes == 8 ? static_cast<const int64_t*>(p.drafted)[at] : static_cast<const int32_t*>(p.drafted)[at];
}
template <typename T>
__device__ __forceinline__ const typename T::Store* target_row(const VerifyParams& p, int b, int i)
{
    return static_cast<const typename T::Store*>(p.x) + b * p.stride_b + i * p.stride_t;
}
template <typename T>
__device__ __forceinline__ const typename T::Store* draft_row(const VerifyParams& p, int b, int i)
{
    return static_cast<const typename T::Store*>(p.draft) + b * p.draft_stride_b + i * p.draft_stride_t;
}

// Values in an order of whole numbers, equal ones by index, lowest first.
__device__ __forceinline__ uint64_t key_of(float x, int i)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return (uint64_t)(b >> 31 ? ~b : b | 0x80000000u) << 32 | (uint32_t)~i;
}
__device__ __forceinline__ uint64_t wave_best(uint64_t k)
{
    for (int o = 32; o > 0; o >>= 1) k = max(k, (uint64_t)__shfl_xor((unsigned long long)k, o, 64));
    return k;
}
// A double of another lane of 16 (DPP); 0 where there is none, or the lane's row is masked out.
template <int Control, int Rows>
__device__ __forceinline__ double from_lane(double v)
{
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), Control, Rows, 0xf, Rows == 0xf);
    const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), Control, Rows, 0xf, Rows == 0xf);
    return __hiloint2double(hi, lo);
}
__device__ __forceinline__ double lane_of(double v, int lane)
{
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}
// The sum over a wave, in every lane.
__device__ __forceinline__ double wave_sum(double v)
{
    v += from_lane<0x128, 0xf>(v);  // rotated by 8, 4, 2, 1
    v += from_lane<0x124, 0xf>(v);
    v += from_lane<0x122, 0xf>(v);
    v += from_lane<0x121, 0xf>(v);
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
// The sums of the lanes up to each.
__device__ __forceinline__ double wave_scan(double v)
{
    v += from_lane<0x111, 0xf>(v);  // moved up by 1, 2, 4, 8 within 16 lanes
    v += from_lane<0x112, 0xf>(v);
    v += from_lane<0x114, 0xf>(v);
    v += from_lane<0x118, 0xf>(v);
    v += from_lane<0x142, 0xa>(v);  // a row's last lane to the row behind it: rows 1 and 3
    v += from_lane<0x143, 0xc>(v);  // lane 31 to rows 2 and 3
    return v;
}

// exp(scale (x - m)) for x <= m, in 64 bits: the place where a running sum passes a random number shows errors of 32. With t
// its logarithm of base 2, n the whole number next to t and f = t - n, 2^f is the polynomial of degree 8 that meets it at the
// nine Chebyshev points of [-1/2, 1/2] (1.1e-12 off at most); n is added to the exponent. 0 for t <= -1,000, -inf among it.
struct Weights {
    double m, scale2;
    double c[8];  // of the polynomial, in scalar registers (otherwise the compiler moves a constant for every product)
    __device__ __forceinline__ Weights(float top, float scale) : m(top), scale2((double)scale * 1.44269504088896340736)
    {
        const double of[8] = {6.931471805459335e-01,  2.402265069581299e-01,  5.550410941205933e-02,  9.618129159402558e-03,
                              1.3333450568000645e-03, 1.5403455852453838e-04, 1.5310079402249296e-05, 1.3255224878668817e-06};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            c[k] = of[k];
            asm("" : "+s"(c[k]));
        }
    }
    // (of a NaN one without a sign, whatever that of x)
    __device__ __forceinline__ double log2_of(float x) const { return fabs((double)x - m) * -scale2; }
    __device__ __forceinline__ double exp2_of(double t) const
    {
        const double shifted = t + 6755399441055744.;  // 1.5 * 2^52: whole numbers in the last bits
        const double f = t - (shifted - 6755399441055744.);
        double e = fma(f, c[7], c[6]);
#pragma unroll
        for (int k = 5; k >= 0; --k) e = fma(e, f, c[k]);
        e = fma(e, f, 1.);
        return __hiloint2double(__double2hiint(e) + (__double2loint(shifted) << 20), __double2loint(e));
    }
    __device__ __forceinline__ double operator()(float x) const
    {
        const double t = log2_of(x);
        return t > -1000. ? exp2_of(t) : 0.;
    }
};

// 2^(j / 64)
struct Roots {
    double of[64];
};
constexpr Roots make_roots()
{
    const double root[6] = {1.0108892860517005, 1.0218971486541166, 1.0442737824274138,
                            1.0905077326652577, 1.189207115002721,  1.4142135623730951};  // of 2: the 64th, 32nd and so on
    Roots r{};
    for (int j = 0; j < 64; ++j) {
        r.of[j] = 1.;
        for (int b = 0; b < 6; ++b)
            if (j >> b & 1) r.of[j] *= root[b];
    }
    return r;
}
__device__ const Roots kRoots = make_roots();

// The same exponential for code that all 64 lanes of a wave go through: 64 t is rounded to a whole number 64 n + j, lane j holds
// 2^(j / 64), and 2^f for |f| <= 1/128 is 1 and a polynomial of degree 3 (6.2e-12 off at most). 13 operations of the vector pipe
// and two passes through the crossbar for a logit, where degree 8 has 17. Lanes ask for two logits' roots before they use one (33 us
// for the rows below; one 34, four 33 with registers for a wave less).
constexpr int kAtOnce = 2;
struct WaveWeights {
    double m, scale2, c[3];
    int hi, lo;  // of the lane's root, less j in the place to which j is shifted
    __device__ __forceinline__ explicit WaveWeights(double root)
    {
        const double of[3] = {0.6931471805578869, 0.24022699328385197, 0.05550422379655395};
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            c[k] = of[k];
            asm("" : "+s"(c[k]));
        }
        hi = __double2hiint(root) - (int)((threadIdx.x & 63) << 14);
        lo = __double2loint(root);
    }
    __device__ __forceinline__ void against(float top, float scale)
    {
        m = top;
        scale2 = (double)scale * 1.44269504088896340736;
    }
    static __device__ __forceinline__ double root() { return kRoots.of[threadIdx.x & 63]; }
    // t = log2 of the weight, at least -1,000: its parts on their way, then s + 2^t
    struct Asked {
        double f;
        int j, high, low;
    };
    __device__ __forceinline__ Asked ask(double t) const
    {
        const double shifted = t + 105553116266496.;  // 1.5 * 2^46: 64ths in the last bits
        const int j = __double2loint(shifted);
        return {t - (shifted - 105553116266496.), j, __builtin_amdgcn_ds_bpermute(j << 2, hi), __builtin_amdgcn_ds_bpermute(j << 2, lo)};
    }
    __device__ __forceinline__ double add(const Asked& a, double s) const
    {
        double e = fma(a.f, c[2], c[1]);
        e = fma(e, a.f, c[0]);
        e = fma(e, a.f, 1.);
        return fma(__hiloint2double(a.high + (a.j << 14), a.low), e, s);
    }
    __device__ __forceinline__ double log2_of(float x) const { return fabs((double)x - m) * -scale2; }
    // 2^-1000 where it is to be 0, which adds nothing beside the 1 of the largest: t's high word is made at most that of
    // -1,000, as a whole number without a sign, where a NaN's is smaller. A NaN, and a +inf, which is the m then, come out as a
    // NaN. (A comparison of every logit for that: 6 us more for 43 million.)
    template <int N>
    __device__ __forceinline__ double add_at_least(const float* x, double s) const
    {
        Asked a[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const double t = log2_of(x[k]);
            a[k] = ask(__hiloint2double((int)min((uint32_t)__double2hiint(t), 0xc08f4000u), __double2loint(t)));
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < N; ++k) s = add(a[k], s);
        return s;
    }
    __device__ __forceinline__ double operator()(float x) const
    {
        const double t = log2_of(x), e = add(ask(fmax(t, -1000.)), 0.);
        return t > -1000. ? e : 0.;
    }
};

// A lane's logits of a part: chunks first, first + Threads and on of the row, -inf behind its end.
template <typename T, int Threads, int Chunks>
__device__ __forceinline__ void load_part(const typename T::Store* x, int first, int V, float (*f)[8])
{
    if (V < 8) {
#pragma unroll
        for (int k = 0; k < Chunks; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) f[k][j] = k == 0 && first == 0 && j < V ? T::load(x + j) : -INFINITY;
        return;
    }
    const int last = (V - 1) / 8;
    Raw<T> v[Chunks];
#pragma unroll
    for (int k = 0; k < Chunks; ++k) v[k] = raw_at<T, kAny>(x, min(first + k * Threads, last), V);
#pragma unroll
    for (int k = 0; k < Chunks; ++k) {
        const int c = first + k * Threads;
        v[k].unpack(f[k]);
        if (c < last) continue;
        if (V % 8) unpack_at<T, kAny>(v[k], last, V, f[k]);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c * 8 + j >= V) f[k][j] = -INFINITY;
    }
}

// ---- every row of a sequence's, a part at a time, a wave each, with no word between waves. Bound by the vector pipe, for the most
// part: 19 instructions a logit, 11 of them of 64 bits. 48 sequences of 1 to 7 rows of 128,000 fp16 and as many of the draft's but
// one, 43 million logits: 33 us, of which the instructions fill 20; 38 with the polynomial of degree 8, 17 with no exponentials.
// By counters they fill 81% of the cycles in which a compute unit has a wave, and those are 70% of the kernel's: the rest is its
// beginning and end, and waves of rows that a sequence does not have, nearly half of those that start. 130 sequences of 4
// rows of 50,021 fp32: 20 us and 23, which is what reading them takes.

template <typename T, bool Greedy>
__global__ __launch_bounds__(kThreads) void k_verify_rows(VerifyParams p, SeqLengths lens, int64_t units)
{
    Space space;
    space_of(p.workspace, p.B, p.K, p.parts, &space);
    const int rows = p.draft ? 2 * p.K + 1 : p.K + 1, lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    WaveWeights weight(Greedy ? 0. : WaveWeights::root());
    for (int64_t u = (int64_t)blockIdx.x * kWaves + wave; u < units; u += (int64_t)gridDim.x * kWaves) {
        const int64_t of = u / p.parts;
        const int part = (int)(u - of * p.parts), b = (int)(of / rows), row = (int)(of - (int64_t)b * rows);
        const bool of_draft = row > p.K;
        const int i = of_draft ? row - p.K - 1 : row, n = drafts_of(p, lens, b);
        if (of_draft ? i >= n : i > n) continue;
        const int first = part * (kVerifyPart / 8) + lane;
        float f[kChunks][8];
        load_part<T, 64, kChunks>(of_draft ? draft_row<T>(p, b, i) : target_row<T>(p, b, i), first, p.V, f);
        float m = -INFINITY;
        bool bad = false;
#pragma unroll
        for (int k = 0; k < kChunks; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                m = fmaxf(m, f[k][j]);
                if (Greedy) bad |= !(f[k][j] < INFINITY);
            }
        m = max_over<64>(m);
        double s = 0.;
        uint64_t best = 0;
        if (Greedy) {
            s = m > -INFINITY ? 1. : 0.;
#pragma unroll
            for (int k = 0; k < kChunks; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int at = (first + k * 64) * 8 + j;
                    if (at < p.V) best = max(best, key_of(f[k][j], at));
                }
            best = wave_best(best);
        } else {
            // (of nothing but -inf, and NaN perhaps: against 0)
            weight.against(m > -INFINITY ? m : 0.f, of_draft ? p.draft_scale : p.scale);
#pragma unroll
            for (int k = 0; k < kChunks; ++k) {
                if ((first - lane + k * 64) * 8 >= p.V) break;  // (nothing but padding)
#pragma unroll
                for (int j = 0; j < 8; j += kAtOnce) s = weight.add_at_least<kAtOnce>(f[k] + j, s);
            }
        }
        s = wave_sum(Greedy && bad ? (double)NAN : s);
        if (!Greedy && s < 0x1p-500) s = 0.;  // (nothing but -inf)
        if (lane == 0)
            space.parts[((int64_t)b * (2 * p.K + 1) + row) * p.parts + part] = {s, m, Greedy ? (int)~(uint32_t)best : 0};
    }
}

// ---- which row ends a sequence

struct RowSum {
    float m;
    double s;
    int first, flags;
};

// A wave joins the parts of a row.
template <bool Greedy>
__device__ __forceinline__ RowSum join(const VerifyParams& p, const Space& space, int b, int row, float scale)
{
    const Part* part = space.parts + ((int64_t)b * (2 * p.K + 1) + row) * p.parts;
    const int lane = threadIdx.x & 63;
    const Part own = lane < p.parts ? part[lane] : Part{0., -INFINITY, 0};
    float m = own.m;
    for (int k = lane + 64; k < p.parts; k += 64) m = fmaxf(m, part[k].m);
    m = max_over<64>(m);
    const Weights weight(m == -INFINITY ? 0.f : m, scale);
    double s = 0.;
    uint64_t best = 0;
    const auto add = [&](const Part& q) {
        s += q.s * weight(q.m);
        if (Greedy) best = max(best, key_of(q.m, q.first));
    };
    if (lane < p.parts) add(own);
    for (int k = lane + 64; k < p.parts; k += 64) add(part[k]);
    s = wave_sum(s);
    if (Greedy) best = wave_best(best);
    return {m, s, Greedy ? (int)~(uint32_t)best : 0, !(s < INFINITY) ? 2 : m == -INFINITY ? 1 : 0};
}

// The first row that ends sequence b, by a whole workgroup, a wave a row: the first drafted token that is not taken, or the
// row behind the last.
template <typename T, bool Greedy>
__device__ __forceinline__ Choice choose(const VerifyParams& p, const Space& space, int b, int n, int* ends, Choice* shared)
{
    if (threadIdx.x == 0) *ends = n;
    __syncthreads();
    const int waves = blockDim.x >> 6;
    Choice c{-1, 0, kAll, -1, 0.f, 0.f, 0., 0.};
    for (int i = threadIdx.x >> 6; i <= n; i += waves) {
        const int64_t d = i < n ? drafted(p, b, i) : 0;
        const bool known = d >= 0 && d < p.V, two = !Greedy && p.draft && i < n;
        // (all that the row takes is on its way before any of it is waited for)
        const float u = !Greedy && i < n ? p.uniforms[(int64_t)b * (p.K + 1) + i] : 0.f;
        const float xd = !Greedy && known ? T::load(target_row<T>(p, b, i) + d) : 0.f;
        const float yd = two && known ? T::load(draft_row<T>(p, b, i) + d) : 0.f;
        const RowSum r = join<Greedy>(p, space, b, i, p.scale);
        RowSum q{0.f, 1., 0, 0};
        if (two) q = join<false>(p, space, b, p.K + 1 + i, p.draft_scale);
        const int flags = r.flags | q.flags | (known ? 0 : 4);
        bool ok = i < n && flags == 0;
        const double per = 1. / r.s, per_q = 1. / q.s;
        if (ok && Greedy) ok = d == r.first;
        if (ok && !Greedy) {
            const double e = Weights(r.m, p.scale)(xd), eq = two ? Weights(q.m, p.draft_scale)(yd) : 1.;
            const double here = e / r.s, there = u * (eq / q.s);
            ok = there < here;
        }
        if (ok) continue;
        c = {i, flags, flags ? kLost : i == n ? kAll : two ? kDrafted : kGiven, Greedy ? r.first : (int)d, r.m, q.m, per, per_q};
        if ((threadIdx.x & 63) == 0) atomicMin(ends, i);
        break;
    }
    __syncthreads();
    if (c.row == *ends && (threadIdx.x & 63) == 0) *shared = c;
    __syncthreads();
    return *shared;
}

__device__ __forceinline__ void write_tokens(const VerifyParams& p, int b, const Choice& c, int token)
{
    for (int i = threadIdx.x; i <= p.K; i += blockDim.x)
        p.tokens[(int64_t)b * (p.K + 1) + i] = i < c.row ? (int)drafted(p, b, i) : i == c.row ? token : -1;
    if (threadIdx.x > 0) return;
    p.accepted[b] = c.row;
    if (p.status) p.status[b] = c.flags;
}

template <typename T>
__global__ __launch_bounds__(kPickThreads) void k_verify_greedy(VerifyParams p, SeqLengths lens)
{
    __shared__ int ends;
    __shared__ Choice shared;
    Space space;
    space_of(p.workspace, p.B, p.K, p.parts, &space);
    for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
        const Choice c = choose<T, true>(p, space, b, drafts_of(p, lens, b), &ends, &shared);
        write_tokens(p, b, c, c.kind == kLost ? -1 : c.token);
        __syncthreads();
    }
}

// What is left of p - q, for all 64 lanes of a wave. The sums of the parts and the token in one of them both go by this: where
// p and q are the same but for rounding, another exponential leaves nothing of a part that has been chosen for what this one
// leaves. (Equal products have to leave nothing: no product goes unrounded into the difference.)
struct LeftOver {
    WaveWeights p, q;
    double per, per_q;
    __device__ __forceinline__ LeftOver(double root, const VerifyParams& v, const Choice& c) : p(root), q(root), per(c.per), per_q(c.per_q)
    {
        p.against(c.m, v.scale);
        q.against(c.mq, v.draft_scale);
    }
    __device__ __forceinline__ double operator()(float x, float y) const
    {
#pragma clang fp contract(off)
        const double a = p(x) * per, b = q(y) * per_q;
        return fmax(0., a - b);
    }
};

// The sum over a workgroup, the same bits in every thread. `parts`: a place for each wave.
__device__ __forceinline__ double block_sum(double v, double* parts)
{
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) v += parts[w];
    return v;
}

// The row that ends every sequence, where a draft's logits are given: 5 us for 48 sequences, waits for all but a few operations.
// (In every workgroup of k_verify_rest by itself: 21 us both together, now 17; of one sequence 12 and 10.)
template <typename T>
__global__ __launch_bounds__(kPickThreads) void k_verify_choose(VerifyParams p, SeqLengths lens)
{
    __shared__ int ends;
    __shared__ Choice shared;
    Space space;
    space_of(p.workspace, p.B, p.K, p.parts, &space);
    for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
        const Choice c = choose<T, false>(p, space, b, drafts_of(p, lens, b), &ends, &shared);
        if (threadIdx.x == 0) space.choice[b] = c;
    }
}

// If a drafted token is replaced: the sums of max(0, p - q) of kRestParts parts, two waves each. 11 us for 48 rows of 128,000
// and as many of the draft's, the exponentials' operations as above.
template <typename T>
__global__ __launch_bounds__(kRestThreads) void k_verify_rest(VerifyParams p, int64_t units)
{
    __shared__ double halves[kRestThreads / 64];
    Space space;
    space_of(p.workspace, p.B, p.K, p.parts, &space);
    const int groups = (p.parts + kRestParts - 1) / kRestParts, lane = threadIdx.x & 63, wave = (int)(threadIdx.x >> 6);
    const double root = WaveWeights::root();
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int b = (int)(u / groups), part = (int)(u - (int64_t)b * groups) * kRestParts + wave / 2;
        const Choice c = space.choice[b];
        if (c.kind != kDrafted) continue;
        if (part < p.parts) {
            constexpr int kHalf = kChunks / 2;
            const int first = part * (kVerifyPart / 8) + (wave & 1) * kHalf * 64 + lane;
            float f[kHalf][8], g[kHalf][8];
            load_part<T, 64, kHalf>(target_row<T>(p, b, c.row), first, p.V, f);
            load_part<T, 64, kHalf>(draft_row<T>(p, b, c.row), first, p.V, g);
            const LeftOver left_over(root, p, c);
            double s = 0.;
#pragma unroll
            for (int k = 0; k < kHalf; ++k) {
                if ((first - lane + k * 64) * 8 >= p.V) break;
#pragma unroll
                for (int j = 0; j < 8; ++j) s += left_over(f[k][j], g[k][j]);
            }
            s = wave_sum(s);
            if (lane == 0) halves[wave] = s;
        }
        __syncthreads();
        if (part < p.parts && (threadIdx.x & 127) == 0)
            space.rest[(int64_t)b * p.parts + part] = halves[wave] + halves[wave + 1];
        __syncthreads();
    }
}

// The last token of every sequence: the first whose running sum passes the random number times the whole. Chosen: k_verify_choose
// has said which row ends the sequence. Running sums of the parts, then of the tokens of one; 9 us of waits one after the other
// (10 for 48 sequences; 12 where it also says which row).
template <typename T, bool Chosen>
__global__ __launch_bounds__(kPickThreads) void k_verify_pick(VerifyParams p, SeqLengths lens)
{
    __shared__ double scan[kPickThreads / 64];
    __shared__ int ends, found, last;
    __shared__ Choice shared;
    Space space;
    space_of(p.workspace, p.B, p.K, p.parts, &space);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const double root = Chosen ? WaveWeights::root() : 0.;
    for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
        const float u = p.uniforms[(int64_t)b * (p.K + 1) + p.K];
        Choice c = Chosen ? space.choice[b] : choose<T, false>(p, space, b, drafts_of(p, lens, b), &ends, &shared);
        if (threadIdx.x == 0) {
            found = INT32_MAX;
            last = -1;
        }
        if (c.kind == kLost) {
            write_tokens(p, b, c, -1);
            continue;
        }
        const Weights weight(c.m, p.scale);
        const LeftOver left_over(root, p, c);
        const Part* parts = space.parts + ((int64_t)b * (2 * p.K + 1) + c.row) * p.parts;
        const double* rest = space.rest + (int64_t)b * p.parts;
        // a lane's weights of eight tokens of a part (by whole waves)
        const auto weights_of = [&](int part, double* w) {
            double s = 0.;
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = 0.;
            if (threadIdx.x >= kVerifyPart / 8) return s;
            const int chunk = part * (kVerifyPart / 8) + (int)threadIdx.x;
            float f[1][8], g[1][8];
            load_part<T, 1, 1>(target_row<T>(p, b, c.row), chunk, p.V, f);
            if (Chosen && c.kind == kDrafted) load_part<T, 1, 1>(draft_row<T>(p, b, c.row), chunk, p.V, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                w[j] = Chosen && c.kind == kDrafted ? left_over(f[0][j], g[0][j]) : weight(f[0][j]);
                if (c.kind == kGiven && chunk * 8 + j == c.token) w[j] = 0.;
                s += w[j];
            }
            return s;
        };
        // the part that a token is taken out of is added up again without it: of a sum minus nearly all of it little is right
        double w[8], without = 0.;
        const int given = c.kind == kGiven ? c.token / kVerifyPart : -1;
        if (given >= 0) {
            without = block_sum(weights_of(given, w), scan);
            __syncthreads();
        }
        const auto weight_of = [&](int k) {
            return k >= p.parts ? 0. : Chosen && c.kind == kDrafted ? rest[k] : k == given ? without : parts[k].s * weight(parts[k].m);
        };
        // every wave: running sums of the parts, 64 at a time, and the part that passes
        double whole = 0.;
        for (int k = 0; k < p.parts; k += 64) whole += lane_of(wave_scan(weight_of(k + lane)), 63);
        int out = given;
        if (!(whole > 0.)) {  // nothing is left where p and q are the same but for rounding: p is drawn from
            c.kind = kAll;
            out = -1;
            whole = 0.;
            for (int k = 0; k < p.parts; k += 64)
                whole += lane_of(wave_scan(k + lane < p.parts ? parts[k + lane].s * weight(parts[k + lane].m) : 0.), 63);
        }
        const auto drawn_of = [&](int k) {
            return c.kind != kAll ? weight_of(k) : k >= p.parts ? 0. : parts[k].s * weight(parts[k].m);
        };
        const double mark = (double)u * whole;
        double before = 0., run = 0.;
        int part = -1;
        for (int k = 0; k < p.parts && part < 0; k += 64) {
            const double here = drawn_of(k + lane), upto = run + wave_scan(here);
            const uint64_t passed = __ballot(here > 0. && upto > mark);
            if (passed) {
                const int at = __ffsll((unsigned long long)passed) - 1;
                part = k + at;
                before = at > 0 ? lane_of(upto, at > 0 ? at - 1 : 0) : run;
            }
            run = lane_of(upto, 63);
        }
        if (part < 0) {  // a number of 1 or more: the last token of any weight
            for (int k = 0; k < p.parts; k += 64) {
                const uint64_t some = __ballot(drawn_of(k + lane) > 0.);
                if (some) part = k + 63 - __clzll((long long)some);
            }
            before = -INFINITY;
        }
        double sum = 0.;
        if (part == out)
            for (int j = 0; j < 8; ++j) sum += w[j];
        else
            sum = weights_of(part, w);
        const double upto = wave_scan(sum);
        if (lane == 63) scan[wave] = upto;
        __syncthreads();
        double cum = before;
        for (int k = 0; k < wave; ++k) cum += scan[k];
        cum += upto - sum;
        const int first = part * kVerifyPart + (int)threadIdx.x * 8;
        int mine = INT32_MAX, some = -1;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            cum += w[j];
            if (w[j] > 0.) {
                some = first + j;
                if (cum > mark && mine == INT32_MAX) mine = first + j;
            }
        }
        if (mine != INT32_MAX) atomicMin(&found, mine);
        if (some >= 0) atomicMax(&last, some);
        __syncthreads();
        write_tokens(p, b, c, found != INT32_MAX ? found : last);
        __syncthreads();
    }
}

}  // namespace

size_t verify_workspace(int64_t B, int K, int V)
{
    return space_of(nullptr, B, K, (V + kVerifyPart - 1) / kVerifyPart, nullptr);
}

hipError_t launch_verify(const VerifyParams& p, const SeqLengths& lens, int dtype, hipStream_t stream)
{
    const int rows = p.draft ? 2 * p.K + 1 : p.K + 1;
    const int64_t all = ((int64_t)p.B * rows * p.parts + kWaves - 1) / kWaves, units = (int64_t)p.B * rows * p.parts;
    const int64_t groups = (int64_t)p.B * ((p.parts + kRestParts - 1) / kRestParts);
    const auto grid_of = [](int64_t n) { return (int)std::min<int64_t>(n, 1 << 20); };
    by_type(dtype, [&](auto type) {
        using T = decltype(type);
        if (!p.uniforms) {
            k_verify_rows<T, true><<<grid_of(all), kThreads, 0, stream>>>(p, lens, units);
            k_verify_greedy<T><<<grid_of(p.B), kPickThreads, 0, stream>>>(p, lens);
            return;
        }
        k_verify_rows<T, false><<<grid_of(all), kThreads, 0, stream>>>(p, lens, units);
        if (p.draft) {
            k_verify_choose<T><<<grid_of(p.B), kPickThreads, 0, stream>>>(p, lens);
            k_verify_rest<T><<<grid_of(groups), kRestThreads, 0, stream>>>(p, groups);
            k_verify_pick<T, true><<<grid_of(p.B), kPickThreads, 0, stream>>>(p, lens);
        } else {
            k_verify_pick<T, false><<<grid_of(p.B), kPickThreads, 0, stream>>>(p, lens);
        }
    });
    return hipGetLastError();
}

}  // namespace lfmmi
