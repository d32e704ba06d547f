// Log probabilities of given tokens, with entropy and the best alternatives of every row of
// logits, and their gradient. See include/lfmmi.h for the formulas.
#include <hip/hip_runtime.h>

#include "../../include/lfmmi.h"
#include "operators.h"

namespace lfmmi {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.693147180559945309f;
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

struct F32 {
    using Store = float;
    static __device__ float load(const Store* p) { return *p; }
    static __device__ void store(Store* p, float v) { *p = v; }
};
struct Bf16 {
    using Store = uint16_t;
    static __device__ float load(const Store* p) { return __uint_as_float((uint32_t)*p << 16); }
    static __device__ void store(Store* p, float v)
    {
        const __bf16 r = (__bf16)v;  // to nearest, ties to even
        *p = __builtin_bit_cast(uint16_t, r);
    }
};
struct F16 {
    using Store = _Float16;
    static __device__ float load(const Store* p) { return (float)*p; }
    static __device__ void store(Store* p, float v) { *p = (_Float16)v; }
};

// What a lane, a wave and a workgroup know of the logits they have read: the largest of them,
// and over all of them, with y = (x - m) * scale * log2(e), the sums of 2^y and of y 2^y.
struct Sums {
    float m, s, u;
};

// m starts at the lowest finite value, not at -inf: differences to it are then never
// (-inf) - (-inf), and a row of nothing but -inf ends with s == 0. A row of nothing but the
// type's lowest value is a uniform one.
__device__ __forceinline__ Sums no_sums() { return {-3.402823466e38f, 0.f, 0.f}; }

// Sums taken against m, as they are against `to` >= m.
__device__ __forceinline__ void shift(Sums& a, float to, float scale2)
{
    // (the difference can overflow to -inf: clamped, so that 0 * -inf does not arise)
    const float dy = fmaxf((a.m - to) * scale2, -1e30f);
    const float f = exp2f(dy);
    a.u = f * (a.u + dy * a.s);
    a.s *= f;
    a.m = to;
}

__device__ __forceinline__ Sums join(Sums a, Sums b, float scale2)
{
    const float to = fmaxf(a.m, b.m);
    shift(a, to, scale2);
    shift(b, to, scale2);
    return {to, a.s + b.s, a.u + b.u};
}

__device__ __forceinline__ void add(Sums& a, float x, float scale2)
{
    if (x > a.m) shift(a, x, scale2);
    const float y = (x - a.m) * scale2, e = exp2f(y);
    a.s += e;
    a.u += e * fmaxf(y, -1e30f);  // (0 * -inf does not arise; a NaN stays in e)
}

// Values in an order of whole numbers, equal ones (-0 and 0 are) by index, lowest first.
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

// Everything but the alternatives, by one lane.
__device__ void write_row(const TokenParams& p, int64_t row, const Row& r, const Sums& a,
                          float x_target, float* m_out, float* logs_out)
{
    int flags = 0;
    float logp = 0.f, entropy = 0.f, m = 0.f, logs = 0.f;
    if (r.live) {
        m = a.m;
        const float log2s = log2f(a.s);
        logs = log2s * kLn2;
        if (!(a.s < INFINITY)) {  // NaN; an inf - inf on the way
            flags = 2;
            m = logs = logp = entropy = NAN;
        } else if (a.s == 0.f) {
            flags = 1;
            logp = -INFINITY;
            m = logs = -INFINITY;
        } else {
            entropy = kLn2 * (log2s - a.u / a.s);
            logp = (x_target - m) * p.scale - logs;
        }
        if (r.target >= p.V) {
            flags |= 4;
            logp = NAN;
        }
    }
    if (p.logp) p.logp[row] = logp;
    if (p.entropy) p.entropy[row] = entropy;
    if (p.stats) {
        p.stats[2 * row] = m;
        p.stats[2 * row + 1] = logs;
    }
    if (p.status) p.status[row] = flags;
    *m_out = m;
    *logs_out = logs;
}

__device__ void write_top(const TokenParams& p, int64_t row, int k, uint64_t key, bool live,
                          float m, float logs)
{
    const int64_t at = row * p.top_k + k;
    const bool bad = m != m;
    if (p.top_id) p.top_id[at] = live && !bad ? index_of(key) : -1;
    if (p.top_logp)
        p.top_logp[at] = !live ? 0.f : m == -INFINITY ? -INFINITY : (value_of(key) - m) * p.scale - logs;
}

__device__ __forceinline__ uint64_t wave_max_key(uint64_t k)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const uint64_t other = __shfl_xor(k, o, 64);
        k = other > k ? other : k;
    }
    return k;
}

// One workgroup a row: one pass for the sums, then one for each alternative.
template <typename D>
__global__ __launch_bounds__(kThreads) void k_token_rows(TokenParams p, SeqLengths lens)
{
    using Store = typename D::Store;
    __shared__ Sums parts[kWaves];
    __shared__ uint64_t keys[kWaves];
    __shared__ float row_m, row_logs;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float scale2 = p.scale * kLog2e;
    const int64_t rows = (int64_t)p.B * p.T;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const int b = (int)(row / p.T), t = (int)(row % p.T);
        const Row r = row_of(p, lens, b, t);
        const Store* x = static_cast<const Store*>(p.x) + b * p.stride_b + t * p.stride_t;
        Sums a = no_sums();
        if (r.live)
            for (int i = threadIdx.x; i < p.V; i += kThreads) add(a, D::load(x + i), scale2);
        for (int o = 32; o > 0; o >>= 1)
            a = join(a, {__shfl_xor(a.m, o, 64), __shfl_xor(a.s, o, 64), __shfl_xor(a.u, o, 64)}, scale2);
        if (lane == 0) parts[wave] = a;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kWaves; ++w) a = join(a, parts[w], scale2);
            const float xt = r.live && r.target >= 0 && r.target < p.V ? D::load(x + r.target) : 0.f;
            write_row(p, row, r, a, xt, &row_m, &row_logs);
        }
        __syncthreads();
        uint64_t last = ~0ull;
        for (int k = 0; k < p.top_k; ++k) {
            uint64_t best = 0;
            if (r.live)
                for (int i = threadIdx.x; i < p.V; i += kThreads) {
                    const uint64_t key = key_of(D::load(x + i), i);
                    if (key < last && key > best) best = key;
                }
            best = wave_max_key(best);
            if (lane == 0) keys[wave] = best;
            __syncthreads();
            for (int w = 0; w < kWaves; ++w) best = keys[w] > best ? keys[w] : best;
            if (threadIdx.x == 0) write_top(p, row, k, best, r.live, row_m, row_logs);
            last = best;
            __syncthreads();
        }
    }
}

template <typename D>
__global__ __launch_bounds__(kThreads) void k_token_grad(TokenGradParams p, SeqLengths lens)
{
    using Store = typename D::Store;
    const int64_t rows = (int64_t)p.B * p.T;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const int b = (int)(row / p.T), t = (int)(row % p.T);
        const Row r = row_of(p, lens, b, t);
        const Store* x = static_cast<const Store*>(p.x) + b * p.stride_b + t * p.stride_t;
        Store* out = static_cast<Store*>(p.grad) + row * p.V;
        const float m = p.stats[2 * row], logs = p.stats[2 * row + 1];
        const bool zero = !r.live || !(m > -INFINITY) || r.target >= p.V;
        const float g = p.grad_logp ? p.grad_logp[row] * p.scale : 0.f;
        const float h = p.grad_entropy ? p.grad_entropy[row] * p.scale : 0.f;
        const float c = h != 0.f ? g + h * p.entropy[row] : g;
        for (int i = threadIdx.x; i < p.V; i += kThreads) {
            float v = 0.f;
            if (!zero) {
                const float l = fmaxf((D::load(x + i) - m) * p.scale - logs, -1e4f);
                const float pr = exp2f(l * kLog2e);
                v = -pr * (c + h * l);
                if (i == r.target) v = -g * expm1f(l) - pr * (c - g + h * l);
            }
            D::store(out + i, v);
        }
    }
}

}  // namespace

hipError_t launch_token_logprobs(const TokenParams& p, const SeqLengths& lens, int dtype,
                                 hipStream_t stream)
{
    const int64_t rows = (int64_t)p.B * p.T;
    const dim3 grid((unsigned)(rows < (1 << 20) ? rows : 1 << 20));
    if (dtype == LFMMI_F32)
        k_token_rows<F32><<<grid, kThreads, 0, stream>>>(p, lens);
    else if (dtype == LFMMI_BF16)
        k_token_rows<Bf16><<<grid, kThreads, 0, stream>>>(p, lens);
    else
        k_token_rows<F16><<<grid, kThreads, 0, stream>>>(p, lens);
    return hipGetLastError();
}

size_t token_workspace(int, int64_t, int, int) { return 0; }

hipError_t launch_token_grad(const TokenGradParams& p, const SeqLengths& lens, int dtype,
                             hipStream_t stream)
{
    const int64_t rows = (int64_t)p.B * p.T;
    const dim3 grid((unsigned)(rows < (1 << 20) ? rows : 1 << 20));
    if (dtype == LFMMI_F32)
        k_token_grad<F32><<<grid, kThreads, 0, stream>>>(p, lens);
    else if (dtype == LFMMI_BF16)
        k_token_grad<Bf16><<<grid, kThreads, 0, stream>>>(p, lens);
    else
        k_token_grad<F16><<<grid, kThreads, 0, stream>>>(p, lens);
    return hipGetLastError();
}

}  // namespace lfmmi
