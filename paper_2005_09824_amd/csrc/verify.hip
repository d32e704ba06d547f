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

constexpr float kLog2e = 1.44269504088896341f;
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kChunks = kVerifyPart / 8 / kThreads;  // of eight logits, that a lane takes of a part
constexpr int kPickThreads = kVerifyPart / 8;

// What a part of a row comes to: its largest logit m, the sum of 2^((x - m) scale log2 e) (NaN where a logit is NaN or
// +inf), the first index of the largest.
struct Part {
    float m, s;
    int first;
};

enum Kind { kLost, kAll, kDrafted, kGiven };  // what the last token is drawn from: nothing, p, p - q, p without the drafted one
struct Choice {
    int row, flags, kind, token;
    float m, mq;
};

struct Space {  // of the workspace
    Part* parts;      // [B, 2 K + 1, parts]: K + 1 rows of the target, K of the draft
    Choice* choice;   // [B]
    double* sums;     // [B, parts]: sums of exponentials of the row that is drawn from
    double* draft;    // [B, parts]: the same of the draft's row
    double* rest;     // [B, parts]: sums of what is drawn from
};
__host__ __device__ size_t up(size_t bytes) { return (bytes + 15) / 16 * 16; }
__host__ __device__ size_t space_of(void* workspace, int64_t B, int K, int parts, Space* s)
{
    char* at = static_cast<char*>(workspace);
    const size_t rows = up((size_t)B * (2 * (size_t)K + 1) * parts * sizeof(Part)), choices = up((size_t)B * sizeof(Choice)),
                 sums = up((size_t)B * parts * sizeof(double));
    if (s) {
        s->parts = reinterpret_cast<Part*>(at);
        s->choice = reinterpret_cast<Choice*>(at + rows);
        s->sums = reinterpret_cast<double*>(at + rows + choices);
        s->draft = reinterpret_cast<double*>(at + rows + choices + sums);
        s->rest = reinterpret_cast<double*>(at + rows + choices + 2 * sums);
    }
    return rows + choices + 3 * sums;
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
__device__ __forceinline__ double wave_sum(double v)
{
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// exp(scale (x - m)), to 64 bits: the place where a running sum passes a random number shows errors of 32.
__device__ __forceinline__ double weight(float x, float m, float scale) { return exp(((double)x - (double)m) * (double)scale); }

// ---- every row of a sequence's, a part at a time

template <typename T, bool Greedy>
__global__ __launch_bounds__(kThreads) void k_verify_rows(VerifyParams p, SeqLengths lens, int64_t units)
{
    __shared__ float parts[2][kWaves];
    __shared__ uint64_t keys[kWaves];
    Space space;
    space_of(p.workspace, p.B, p.K, p.parts, &space);
    const int rows = p.draft ? 2 * p.K + 1 : p.K + 1, wave = threadIdx.x >> 6;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int part = (int)(u % p.parts), row = (int)(u / p.parts % rows), b = (int)(u / p.parts / rows);
        const bool of_draft = row > p.K;
        const int i = of_draft ? row - p.K - 1 : row, n = drafts_of(p, lens, b);
        if (of_draft ? i >= n : i > n) continue;
        const typename T::Store* x = of_draft ? draft_row<T>(p, b, i) : target_row<T>(p, b, i);
        const float scale2 = (of_draft ? p.draft_scale : p.scale) * kLog2e;
        const int first = part * kVerifyPart;
        float f[kChunks][8];
#pragma unroll
        for (int k = 0; k < kChunks; ++k) {
            const int c = first + (k * kThreads + threadIdx.x) * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) f[k][j] = -INFINITY;
            if (c + 8 <= p.V) load_at<T, true>(x, c / 8, p.V, f[k]);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < p.V) f[k][j] = T::load(x + c + j);
        }
        float m = -INFINITY;
#pragma unroll
        for (int k = 0; k < kChunks; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) m = fmaxf(m, f[k][j]);
        m = max_over<64>(m);
        if ((threadIdx.x & 63) == 0) parts[0][wave] = m;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) m = fmaxf(m, parts[0][w]);
        const float against = m == -INFINITY ? 0.f : m;  // (a part of nothing but -inf sums to 0)
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < kChunks; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) s += __builtin_amdgcn_exp2f((f[k][j] - against) * scale2);
        s = sum_over<64>(s);
        if ((threadIdx.x & 63) == 0) parts[1][wave] = s;
        if (Greedy) {
            uint64_t best = 0;
#pragma unroll
            for (int k = 0; k < kChunks; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int c = first + (k * kThreads + threadIdx.x) * 8 + j;
                    if (c < p.V) best = max(best, key_of(f[k][j], c));
                }
            best = wave_best(best);
            if ((threadIdx.x & 63) == 0) keys[wave] = best;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            s = 0.f;
            uint64_t best = 0;
            for (int w = 0; w < kWaves; ++w) {
                s += parts[1][w];
                if (Greedy) best = max(best, keys[w]);
            }
            space.parts[((int64_t)b * (2 * p.K + 1) + row) * p.parts + part] = {m, s, Greedy ? (int)~(uint32_t)best : 0};
        }
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
    float m = -INFINITY;
    for (int k = lane; k < p.parts; k += 64) m = fmaxf(m, part[k].m);
    m = max_over<64>(m);
    const float against = m == -INFINITY ? 0.f : m;
    double s = 0.;
    uint64_t best = 0;
    for (int k = lane; k < p.parts; k += 64) {
        const Part q = part[k];
        s += (double)q.s * (double)__builtin_amdgcn_exp2f((q.m - against) * scale * kLog2e);
        if (Greedy) best = max(best, key_of(q.m, q.first));
    }
    s = wave_sum(s);
    if (Greedy) best = wave_best(best);
    return {m, s, Greedy ? (int)~(uint32_t)best : 0, !(s < INFINITY) ? 2 : m == -INFINITY ? 1 : 0};
}

// The sum of a whole row in 64 bits, by a wave.
template <typename T>
__device__ __noinline__ double sum_again(const typename T::Store* x, int V, float m, float scale)
{
    double s = 0.;
    for (int i = threadIdx.x & 63; i < V; i += 64) s += weight(T::load(x + i), m, scale);
    return wave_sum(s);
}

// Sums of 32 bits are off by at most 2^-24 times some 130: a term exp(d) by 4 |d| + 2, where the mean of |d| is at most ln V,
// and 42 additions. Where u q and p are no further apart than kNear the sums are taken again.
constexpr double kNear = 0x1p-14;

// The first row that ends sequence b, by a whole workgroup: the first drafted token that is not taken, or the row behind
// the last. `token`: the greedy one.
template <typename T, bool Greedy>
__device__ __forceinline__ Choice choose(const VerifyParams& p, const Space& space, int b, int n, int* ends)
{
    if (threadIdx.x == 0) *ends = n;
    __syncthreads();
    const int waves = blockDim.x >> 6;
    for (int i = threadIdx.x >> 6; i < n; i += waves) {
        const RowSum r = join<Greedy>(p, space, b, i, p.scale);
        const int64_t d = drafted(p, b, i);
        bool ok = r.flags == 0 && d >= 0 && d < p.V;
        if (ok && Greedy) ok = d == r.first;
        if (ok && !Greedy) {
            const typename T::Store *x = target_row<T>(p, b, i), *y = p.draft ? draft_row<T>(p, b, i) : x;
            const double u = (double)p.uniforms[(int64_t)b * (p.K + 1) + i], e = weight(T::load(x + d), r.m, p.scale);
            RowSum q{0.f, 1., 0, 0};
            double eq = 1.;
            if (p.draft) {
                q = join<false>(p, space, b, p.K + 1 + i, p.draft_scale);
                eq = weight(T::load(y + d), q.m, p.draft_scale);
            }
            double here = e / r.s, there = u * (eq / q.s);
            if (fabs(here - there) <= kNear * here) {
                here = e / sum_again<T>(x, p.V, r.m, p.scale);
                if (p.draft) there = u * (eq / sum_again<T>(y, p.V, q.m, p.draft_scale));
            }
            ok = q.flags == 0 && there < here;
        }
        if (!ok && (threadIdx.x & 63) == 0) atomicMin(ends, i);
    }
    __syncthreads();
    Choice c{*ends, 0, kAll, -1, 0.f, 0.f};
    const RowSum r = join<Greedy>(p, space, b, c.row, p.scale);
    c.m = r.m;
    c.flags = r.flags;
    c.token = r.first;
    if (c.row < n) {
        const int64_t d = drafted(p, b, c.row);
        if (d < 0 || d >= p.V) c.flags |= 4;
        c.kind = kGiven;
        if (!Greedy && p.draft) {
            const RowSum q = join<false>(p, space, b, p.K + 1 + c.row, p.draft_scale);
            c.flags |= q.flags;
            c.mq = q.m;
            c.kind = kDrafted;
        }
    }
    if (c.flags) c.kind = kLost;
    return c;
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
__global__ __launch_bounds__(kThreads) void k_verify_greedy(VerifyParams p, SeqLengths lens)
{
    __shared__ int ends;
    Space space;
    space_of(p.workspace, p.B, p.K, p.parts, &space);
    for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
        const Choice c = choose<T, true>(p, space, b, drafts_of(p, lens, b), &ends);
        write_tokens(p, b, c, c.kind == kLost ? -1 : c.token);
        __syncthreads();
    }
}

// Sum over a workgroup of kThreads, in thread 0.
__device__ __forceinline__ double block_sum(double v, double* parts)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.;
    for (int w = 0; w < kWaves; ++w) v += parts[w];
    return v;
}

// Calls each(i, x_i) for a lane's logits of a part.
template <typename T, typename F>
__device__ __forceinline__ void of_part(const VerifyParams& p, int part, F&& each)
{
    for (int k = 0; k < kChunks; ++k) {
        const int c = part * kVerifyPart + (k * kThreads + (int)threadIdx.x) * 8;
        for (int j = 0; j < 8; ++j)
            if (c + j < p.V) each(c + j);
    }
}

// The row that ends every sequence, and a part's sums of it.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_verify_sums(VerifyParams p, SeqLengths lens, int64_t units)
{
    __shared__ int ends;
    __shared__ double parts[kWaves];
    Space space;
    space_of(p.workspace, p.B, p.K, p.parts, &space);
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int part = (int)(u % p.parts), b = (int)(u / p.parts);
        const Choice c = choose<T, false>(p, space, b, drafts_of(p, lens, b), &ends);
        if (part == 0 && threadIdx.x == 0) space.choice[b] = c;
        if (c.kind != kLost) {
            const typename T::Store* x = target_row<T>(p, b, c.row);
            const int64_t d = c.kind == kGiven ? drafted(p, b, c.row) : -1;
            double s = 0., without = 0., q = 0.;
            of_part<T>(p, part, [&](int i) {
                const double e = weight(T::load(x + i), c.m, p.scale);
                s += e;
                if (i != d) without += e;
            });
            if (c.kind == kDrafted) {
                const typename T::Store* y = draft_row<T>(p, b, c.row);
                of_part<T>(p, part, [&](int i) { q += weight(T::load(y + i), c.mq, p.draft_scale); });
            }
            s = block_sum(s, parts);
            without = block_sum(without, parts);
            q = block_sum(q, parts);
            if (threadIdx.x == 0) {
                space.sums[u] = s;
                space.rest[u] = without;
                space.draft[u] = q;
            }
        }
        __syncthreads();
    }
}

// Sum of a sequence's parts, the same bits in every wave.
__device__ __forceinline__ double total(const double* sums, int parts)
{
    double s = 0.;
    for (int k = threadIdx.x & 63; k < parts; k += 64) s += sums[k];
    return wave_sum(s);
}

__device__ __forceinline__ double left_over(float x, float m, double s, float scale, float y, float mq, double sq, float scale_q)
{
    return fmax(0., weight(x, m, scale) / s - weight(y, mq, scale_q) / sq);
}

// Where a draft's logits are given: a part's sum of max(0, p - q).
template <typename T>
__global__ __launch_bounds__(kThreads) void k_verify_rest(VerifyParams p, int64_t units)
{
    __shared__ double parts[kWaves];
    Space space;
    space_of(p.workspace, p.B, p.K, p.parts, &space);
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int part = (int)(u % p.parts), b = (int)(u / p.parts);
        const Choice c = space.choice[b];
        if (c.kind != kDrafted) continue;
        const double s = total(space.sums + (int64_t)b * p.parts, p.parts), q = total(space.draft + (int64_t)b * p.parts, p.parts);
        const typename T::Store *x = target_row<T>(p, b, c.row), *y = draft_row<T>(p, b, c.row);
        double r = 0.;
        of_part<T>(p, part, [&](int i) {
            r += left_over(T::load(x + i), c.m, s, p.scale, T::load(y + i), c.mq, q, p.draft_scale);
        });
        r = block_sum(r, parts);
        if (threadIdx.x == 0) space.rest[u] = r;
    }
}

// Sums of the lanes up to each.
__device__ __forceinline__ double wave_scan(double v)
{
    const int lane = threadIdx.x & 63;
    for (int o = 1; o < 64; o <<= 1) {
        const double w = __shfl_up(v, o, 64);
        if (lane >= o) v += w;
    }
    return v;
}

// The last token of every sequence: the first whose running sum passes the random number times the whole.
template <typename T>
__global__ __launch_bounds__(kPickThreads) void k_verify_pick(VerifyParams p)
{
    __shared__ double scan[kPickThreads / 64];
    __shared__ int found, last;
    Space space;
    space_of(p.workspace, p.B, p.K, p.parts, &space);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
        Choice c = space.choice[b];
        if (c.kind == kLost) {
            write_tokens(p, b, c, -1);
            continue;
        }
        const double *sums = space.sums + (int64_t)b * p.parts, *rest = space.rest + (int64_t)b * p.parts;
        const double s = total(sums, p.parts);
        const double q = c.kind == kDrafted ? total(space.draft + (int64_t)b * p.parts, p.parts) : 1.;
        // (nothing is left where p and q are the same but for rounding)
        if (!(total(rest, p.parts) > 0.)) {
            c.kind = kAll;
            rest = sums;
        }
        // every wave: running sums of the parts, 64 at a time, and the part that passes
        double whole = 0.;
        for (int k = 0; k < p.parts; k += 64) whole += __shfl(wave_scan(k + lane < p.parts ? rest[k + lane] : 0.), 63, 64);
        const double mark = (double)p.uniforms[(int64_t)b * (p.K + 1) + p.K] * whole;
        double before = 0., run = 0.;
        int part = -1;
        for (int k = 0; k < p.parts && part < 0; k += 64) {
            const double here = k + lane < p.parts ? rest[k + lane] : 0., upto = run + wave_scan(here);
            const uint64_t passed = __ballot(here > 0. && upto > mark);
            if (passed) {
                const int at = __ffsll((unsigned long long)passed) - 1;
                part = k + at;
                const double earlier = __shfl(upto, at > 0 ? at - 1 : 0, 64);
                before = at > 0 ? earlier : run;
            }
            run = __shfl(upto, 63, 64);
        }
        if (part < 0) {  // a number of 1 or more: the last token of any weight
            for (int k = 0; k < p.parts; k += 64) {
                const uint64_t some = __ballot(k + lane < p.parts && rest[k + lane] > 0.);
                if (some) part = k + 63 - __clzll((long long)some);
            }
            before = -INFINITY;
        }
        const typename T::Store* x = target_row<T>(p, b, c.row);
        const typename T::Store* y = c.kind == kDrafted ? draft_row<T>(p, b, c.row) : x;
        const int64_t d = c.kind == kGiven ? drafted(p, b, c.row) : -1;
        const int first = part * kVerifyPart + (int)threadIdx.x * 8;
        double w[8], sum = 0.;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = first + j;
            w[j] = 0.;
            if (i < p.V && i != d)
                w[j] = c.kind == kDrafted
                    ? left_over(T::load(x + i), c.m, s, p.scale, T::load(y + i), c.mq, q, p.draft_scale)
                    : weight(T::load(x + i), c.m, p.scale);
            sum += w[j];
        }
        const double upto = wave_scan(sum);
        if (threadIdx.x == 0) {
            found = INT32_MAX;
            last = -1;
        }
        if (lane == 63) scan[wave] = upto;
        __syncthreads();
        double cum = before;
        for (int k = 0; k < wave; ++k) cum += scan[k];
        cum += upto - sum;
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
    const int64_t units = (int64_t)p.B * p.parts, all = units * rows;
    const auto grid_of = [](int64_t n) { return (int)std::min<int64_t>(n, 1 << 20); };
    by_type(dtype, [&](auto type) {
        using T = decltype(type);
        if (!p.uniforms) {
            k_verify_rows<T, true><<<grid_of(all), kThreads, 0, stream>>>(p, lens, all);
            k_verify_greedy<T><<<grid_of(p.B), kThreads, 0, stream>>>(p, lens);
            return;
        }
        k_verify_rows<T, false><<<grid_of(all), kThreads, 0, stream>>>(p, lens, all);
        k_verify_sums<T><<<grid_of(units), kThreads, 0, stream>>>(p, lens, units);
        if (p.draft && p.K > 0) k_verify_rest<T><<<grid_of(units), kThreads, 0, stream>>>(p, units);
        k_verify_pick<T><<<grid_of(p.B), kPickThreads, 0, stream>>>(p);
    });
    return hipGetLastError();
}

}  // namespace lfmmi
