// Dropout, and the residual's addition with a root-mean-square norm, forward and backward. See
// include/lfmmi.h for the formulas.
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
constexpr float kE4m3Max = 448.f;
constexpr float kSmaller = 0x1p-80f;            // the square of the largest float times that has an exponent of 96
constexpr float kLeastScale = 1.17549435e-38f;  // 2^-126

// Waves of one workgroup take a row each, or all of them one together.
constexpr int threads_of(int lanes) { return lanes == 64 ? kThreads : lanes; }

// ---- dropout alone. Bound by HBM (16,384 rows of 8,189 bf16, a view: 101 us, 5.3 TB/s; 32,000 of 640 fp32: 28 us, 5.9 TB/s); the
// random bits, ten rounds of two products of 32 bits for eight values, fit beside it.

constexpr int kDropoutChunks = 4;  // of eight values, that a lane takes of a row

template <typename T, Width W>
__global__ __launch_bounds__(kThreads) void k_dropout(DropoutParams p, int lanes_log2, uint32_t pieces, uint32_t units)
{
    using Store = typename T::Store;
    const Dropping drop(p.draw);
    const int lanes = 1 << lanes_log2, lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> lanes_log2;
    const int rows = kThreads >> lanes_log2, chunks = (p.D + 7) / 8;
    for (uint32_t u = blockIdx.x; u < units; u += gridDim.x) {
        const uint32_t group = u / pieces;
        const int64_t row = (int64_t)group * rows + sub;
        if (row >= p.R) continue;
        const Store* x = static_cast<const Store*>(p.x) + row * p.stride_x;
        Store* y = static_cast<Store*>(p.y) + row * p.stride_y;
        const int first = (int)(u - group * pieces) * kDropoutChunks * lanes + lane;
        Raw<T> v[kDropoutChunks];
#pragma unroll
        for (int k = 0; k < kDropoutChunks; ++k) {
            const int c = first + k * lanes;
            if (c < chunks) v[k] = raw_at<T, W>(x, c, p.D);
        }
#pragma unroll
        for (int k = 0; k < kDropoutChunks; ++k) {
            const int c = first + k * lanes;
            if (c >= chunks) continue;
            float f[8];
            unpack_at<T, W>(v[k], c, p.D, f);
            if (drop.threshold > 0) drop.apply((uint32_t)row, (uint32_t)c, f);
            store_at<T, W>(y, c, p.D, f, p.once);
        }
    }
}

// ---- norms

// The sum, or the largest, over the G lanes that take a row.
template <int G, bool Max>
__device__ __forceinline__ float over_row(float v, float* parts)
{
    v = Max ? max_over<64>(v) : sum_over<64>(v);
    if (G == 64) return v;
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
    __syncthreads();
    v = parts[0];
    for (int w = 1; w < G / 64; ++w) v = Max ? fmaxf(v, parts[w]) : v + parts[w];
    return v;
}

__device__ __forceinline__ bool inside(const SeqLengths& lens, uint32_t row, int T)
{
    return lens.n == 0 || (int)(row % (uint32_t)T) < lens.T[row / (uint32_t)T];
}

// Rows (b, t) of an array of strides.
__device__ __forceinline__ int64_t offset_of(uint32_t row, int T, int64_t stride_b, int64_t stride_t)
{
    return (int64_t)(row / (uint32_t)T) * stride_b + (int64_t)(row % (uint32_t)T) * stride_t;
}

template <typename T, Width W>
__device__ __forceinline__ void load_weight(const void* w, bool f32, int c, int D, float* f)
{
    if (!w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = 1.f;
    } else if (f32) {
        load_at<F32, W>(static_cast<const float*>(w), c, D, f);
    } else {
        load_at<T, W>(static_cast<const typename T::Store*>(w), c, D, f);
    }
}

__device__ __forceinline__ void store_bytes(uint8_t* q, int left, const float* f)
{
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
        w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], v, true);
    }
    if (left >= 8) {
        __builtin_memcpy(q, w, 8);
        return;
    }
    const uint32_t rest = left & 4 ? w[1] : w[0];
    if (left & 4) __builtin_memcpy(q, &w[0], 4);
    const uint16_t two = (uint16_t)rest;
    if (left & 2) __builtin_memcpy(q + (left & 4), &two, 2);
    if (left & 1) q[left - 1] = (uint8_t)(left & 2 ? rest >> 16 : rest);
}

// y / scale for the values of a row: times the inverse, less what that is off, so that a quotient halfway between two values of
// e4m3 comes out as that. (16,384 rows of 8,192 bf16: 114 us, 108 without what it is off, 138 with a division a value.) Small
// scales are taken times 2^64, their values too, which loses nothing; over an infinite one finite values are 0.
struct Quotient {
    bool small;
    float by, inverse;
    __device__ __forceinline__ explicit Quotient(float scale) : small(scale < 0x1p-60f)
    {
        const float s = small ? scale * 0x1p64f : scale;
        by = s < INFINITY ? s : 0.f;
        inverse = 1.f / s;
    }
    __device__ __forceinline__ void operator()(float* y) const  // eight of them
    {
        if (__builtin_expect(small, 0))
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] *= 0x1p64f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float q = y[i] * inverse;
            y[i] = fmaf(-fmaf(q, by, -y[i]), inverse, q);
        }
    }
};

// A value as it is kept in the type.
template <typename T>
__device__ __forceinline__ float rounded(float v)
{
    if (T::kVec == 4) return v;
    typename T::Store s;
    T::store(&s, v);
    return T::load(&s);
}

// Which of a workgroup's rows a wave has: the same in all its lanes, and held once.
template <int G>
__device__ __forceinline__ int row_in_group()
{
    return threads_of(G) == G ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / G);
}

// Bits of |y| as whole numbers: the largest of them is a NaN's, if there is one.
__device__ __forceinline__ uint32_t magnitude(float y) { return __float_as_uint(y) & 0x7fffffffu; }

// G lanes take a row, N chunks of eight values each, which stay in registers; N == 0: any number of
// chunks, read again for each pass over the row. Bound by HBM: 16,384 rows of 8,192 bf16, two arrays read and two written, 187
// us, 5.7 TB/s, what a copy takes.
template <typename T, Width W, int G, int N>
__global__ __launch_bounds__(threads_of(G)) void k_norm(NormParams p, SeqLengths lens)
{
    using Store = typename T::Store;
    constexpr int kRows = threads_of(G) / G;
    constexpr int kHeld = N > 0 ? N : 1;
    __shared__ float parts[2][G / 64];
    const Dropping drop(p.draw);
    const int lane = threadIdx.x % G, sub = row_in_group<G>(), chunks = (p.D + 7) / 8;
    const uint32_t rows = (uint32_t)p.B * (uint32_t)p.T;
    for (uint32_t row = blockIdx.x * kRows + sub; row < rows; row += gridDim.x * kRows) {
        const Store* x = static_cast<const Store*>(p.x) + offset_of(row, p.T, p.x_stride_b, p.x_stride_t);
        const Store* res = p.residual
            ? static_cast<const Store*>(p.residual) + offset_of(row, p.T, p.r_stride_b, p.r_stride_t) : nullptr;
        const int64_t at = (int64_t)row * p.D;
        Store* sum = p.sum ? static_cast<Store*>(p.sum) + at : nullptr;
        Store* y = p.y ? static_cast<Store*>(p.y) + at : nullptr;
        uint8_t* q = p.q ? p.q + at : nullptr;
        float h[kHeld][8];
        if (!inside(lens, row, p.T)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) h[0][i] = 0.f;
            for (int c = lane; c < chunks; c += G) {
                if (sum) store_at<T, W>(sum, c, p.D, h[0], p.once);
                if (y) store_at<T, W>(y, c, p.D, h[0], p.once);
                if (q) store_bytes(q + c * 8, p.D - c * 8, h[0]);
            }
            if (lane == 0) {
                if (p.rstd) p.rstd[row] = 0.f;
                if (p.q_scale) p.q_scale[row] = 0.f;
            }
            continue;
        }
        const auto add_up = [&](int c, const Raw<T>& a, const Raw<T>& b, float* f) {
            float r[8];
            unpack_at<T, W>(a, c, p.D, f);
            if (res) unpack_at<T, W>(b, c, p.D, r);
            if (drop.threshold > 0) drop.apply((uint32_t)(p.row + row), (uint32_t)c, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = rounded<T>(res ? f[i] + r[i] : f[i]);
        };
        float s = 0.f;
        if (N > 0) {
            Raw<T> a[kHeld], b[kHeld];  // (all on their way before one is waited for)
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                const int c = lane + k * G;
                a[k] = b[k] = no_values<T>();
                if (c < chunks) {
                    a[k] = raw_at<T, W>(x, c, p.D);
                    if (res) b[k] = raw_at<T, W>(res, c, p.D);
                }
            }
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                const int c = lane + k * G;
                add_up(c, a[k], b[k], h[k]);
                if (c < chunks && sum) store_at<T, W>(sum, c, p.D, h[k], p.once);
#pragma unroll
                for (int i = 0; i < 8; ++i) s = fmaf(h[k][i], h[k][i], s);
            }
        } else {
            for (int c = lane; c < chunks; c += G) {
                add_up(c, raw_at<T, W>(x, c, p.D), res ? raw_at<T, W>(res, c, p.D) : no_values<T>(), h[0]);
                if (sum) store_at<T, W>(sum, c, p.D, h[0], p.once);
#pragma unroll
                for (int i = 0; i < 8; ++i) s = fmaf(h[0][i], h[0][i], s);
            }
        }
        if (G > 64) __syncthreads();  // (the row before has read `parts`)
        s = over_row<G, false>(s, parts[0]);
        float rstd = 1.f / sqrtf(s / (float)p.D + p.eps);
        // squares beyond fp32, unless there is an infinity or a NaN: taken again of smaller values
        if (__builtin_expect(!(s < INFINITY), 0)) {
            s = 0.f;
            if (N > 0) {
#pragma unroll
                for (int k = 0; k < kHeld; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) s = fmaf(h[k][i] * kSmaller, h[k][i] * kSmaller, s);
            } else {
                for (int c = lane; c < chunks; c += G) {
                    load_at<T, W>(sum ? sum : x, c, p.D, h[0]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) s = fmaf(h[0][i] * kSmaller, h[0][i] * kSmaller, s);
                }
            }
            s = over_row<G, false>(s, parts[1]);
            rstd = kSmaller / sqrtf(s / (float)p.D);  // (eps of 1e20 at most is nothing beside a mean of 2e31)
            if (G > 64) __syncthreads();
        }
        if (p.rstd && lane == 0) p.rstd[row] = rstd;
        // (what a lane has written itself is read again: from `sum`, or from x where nothing was added)
        const auto scaled = [&](int c, int k, float* f) {
            float w[8];
            load_weight<T, W>(p.weight, p.weight_f32, c, p.D, w);
            if (N == 0) load_at<T, W>(sum ? sum : x, c, p.D, h[0]);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = h[N > 0 ? k : 0][i] * rstd * w[i];
        };
        uint32_t top = 0;
        if (N > 0) {
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                const int c = lane + k * G;
                if (c >= chunks) continue;
                float f[8];
                scaled(c, k, f);
                if (y) store_at<T, W>(y, c, p.D, f, p.once);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    top = max(top, magnitude(f[i]));
                    h[k][i] = f[i];
                }
            }
        } else {
            for (int c = lane; c < chunks; c += G) {
                float f[8];
                scaled(c, 0, f);
                if (y) store_at<T, W>(y, c, p.D, f, p.once);
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, magnitude(f[i]));
            }
        }
        if (!q) continue;
        // (fmaxf passes a NaN over: the bits are compared as values that are none)
        const bool bad = top > 0x7f800000u;
        const float best = over_row<G, true>(bad ? INFINITY : __uint_as_float(top), parts[1]);
        const float none = over_row<G, true>(bad ? 1.f : 0.f, parts[0]);
        const float scale = none > 0.f ? NAN : fmaxf(best / kE4m3Max, kLeastScale);
        const Quotient over(scale);
        if (p.q_scale && lane == 0) p.q_scale[row] = scale;
        if (N > 0) {
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                const int c = lane + k * G;
                if (c >= chunks) continue;
                over(h[k]);
                store_bytes(q + c * 8, p.D - c * 8, h[k]);
            }
        } else {
            for (int c = lane; c < chunks; c += G) {
                float f[8];
                scaled(c, 0, f);
                over(f);
                store_bytes(q + c * 8, p.D - c * 8, f);
            }
        }
    }
}

// Hides from the compiler what a chunk holds: what has been unpacked from it before is not kept for the next time.
template <typename T>
__device__ __forceinline__ void hide(Raw<T>& v)
{
#pragma unroll
    for (int k = 0; k < 8 / T::kVec; ++k) asm volatile("" : "+v"(v.r[k].x), "+v"(v.r[k].y), "+v"(v.r[k].z), "+v"(v.r[k].w));
}

// The same lanes and chunks; a workgroup adds its rows' share of the weight's gradient up, and leaves it as a
// row of partial sums. Bound by HBM: 16,384 rows of 8,192 bf16, three arrays read and two written, 242 to 269 us, 5.0 to 5.5 TB/s
// (435 without the rows asked for ahead).
template <typename T, Width W, int G, int N>
__global__ __launch_bounds__(threads_of(G)) void k_norm_grad(NormGradParams p, SeqLengths lens)
{
    using Store = typename T::Store;
    constexpr int kRows = threads_of(G) / G;
    constexpr int kHeld = N > 0 ? N : 1;
    __shared__ float parts[G / 64];
    const Dropping drop(p.draw);
    const int lane = threadIdx.x % G, sub = row_in_group<G>(), chunks = (p.D + 7) / 8;
    const uint32_t rows = (uint32_t)p.B * (uint32_t)p.T;
    float dw[kHeld][8];
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[k][i] = 0.f;
    float* partial = p.partials ? p.partials + (int64_t)blockIdx.x * p.D : nullptr;
    if (N == 0 && partial && !p.add)
        for (int c = lane; c < chunks; c += G) store_at<F32, W>(partial, c, p.D, dw[0]);
    const uint32_t stride = gridDim.x * kRows;
    const auto row_of = [&](uint32_t row) {
        return static_cast<const Store*>(p.h) + offset_of(row, p.T, p.stride_b, p.stride_t);
    };
    const auto dy_of = [&](uint32_t row) { return static_cast<const Store*>(p.grad_y) + (int64_t)row * p.D; };
    // What a row begins with is asked for while the row before is dealt with, and the weight is held; four chunks a lane
    // of 512 have no registers for that (16,384 columns, 6,000 rows of fp32: 476 us so, 407 without; of bf16 223 and 225), nor two
    // of 768 in 32 bits and odd widths (9,001 columns, 9,000 rows: 577 and 365; of bf16 184 and 228).
    constexpr bool kAhead = N > 0 && G * N < 2048 && !(T::kVec == 4 && W == kAny && G * N >= 1536);
    Raw<T> h_next[kHeld], y_next[kHeld];
    float rstd_next = 0.f;
    const auto ask = [&](uint32_t row) {
        if (N == 0 || row >= rows || !inside(lens, row, p.T)) return;
        rstd_next = p.rstd[row];
        const Store* hr = row_of(row);
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
            const int c = lane + k * G;
            h_next[k] = y_next[k] = no_values<T>();
            if (c >= chunks) continue;
            h_next[k] = raw_at<T, W>(hr, c, p.D);
            if (p.grad_y) y_next[k] = raw_at<T, W>(dy_of(row), c, p.D);
        }
    };
    float w[kHeld][8];
    if (kAhead) {
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            load_weight<T, W>(p.weight, p.weight_f32, min(lane + k * G, chunks - 1), p.D, w[k]);
        ask(blockIdx.x * kRows + sub);
    }
    for (uint32_t row = blockIdx.x * kRows + sub; row < rows; row += stride) {
        const int64_t at = (int64_t)row * p.D;
        const Store* dsum = p.grad_sum ? static_cast<const Store*>(p.grad_sum) + at : nullptr;
        Store* dx = p.grad_x ? static_cast<Store*>(p.grad_x) + at : nullptr;
        Store* dres = p.grad_residual ? static_cast<Store*>(p.grad_residual) + at : nullptr;
        const auto write = [&](int c, float* f) {
            if (dres) store_at<T, W>(dres, c, p.D, f, p.once);
            if (dx) {
                if (drop.threshold > 0) drop.apply((uint32_t)(p.row + row), (uint32_t)c, f);
                store_at<T, W>(dx, c, p.D, f, p.once);
            }
        };
        if (!inside(lens, row, p.T)) {
            float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (int c = lane; c < chunks; c += G) {
                if (dres) store_at<T, W>(dres, c, p.D, zero, p.once);
                if (dx) store_at<T, W>(dx, c, p.D, zero, p.once);
            }
            if (kAhead) ask(row + stride);
            continue;
        }
        if (N > 0 && !kAhead) ask(row);
        const float rstd = N > 0 ? rstd_next : p.rstd[row];
        // n = h rstd and w dy of a chunk
        const auto take = [&](int c, const Raw<T>& a, const Raw<T>& b, const float* w, float* n, float* g, float* dw) {
            unpack_at<T, W>(a, c, p.D, n);
            unpack_at<T, W>(b, c, p.D, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[i] *= rstd;
                if (dw) dw[i] = fmaf(g[i], n[i], dw[i]);
                g[i] *= w[i];
            }
        };
        float n[8], g[8], s = 0.f;
        // (rows stay as they lie in memory, half the registers of their values: they are unpacked twice)
        Raw<T> a[kHeld], b[kHeld], d[kHeld];
        if (N > 0) {
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                const int c = lane + k * G;
                a[k] = h_next[k];
                b[k] = y_next[k];
                d[k] = no_values<T>();
                if (c < chunks && dsum) d[k] = raw_at<T, W>(dsum, c, p.D);
            }
            if (kAhead) ask(row + stride);
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                if (!kAhead) load_weight<T, W>(p.weight, p.weight_f32, min(lane + k * G, chunks - 1), p.D, w[k]);
                take(lane + k * G, a[k], b[k], w[k], n, g, dw[k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) s = fmaf(g[i], n[i], s);
            }
        } else {
            for (int c = lane; c < chunks; c += G) {
                float add[8];
                if (partial) load_at<F32, W>(partial, c, p.D, add);
                load_weight<T, W>(p.weight, p.weight_f32, c, p.D, w[0]);
                take(c, raw_at<T, W>(row_of(row), c, p.D),
                     p.grad_y ? raw_at<T, W>(dy_of(row), c, p.D) : no_values<T>(), w[0], n, g, partial ? add : nullptr);
                if (partial) store_at<F32, W>(partial, c, p.D, add);
#pragma unroll
                for (int i = 0; i < 8; ++i) s = fmaf(g[i], n[i], s);
            }
        }
        if (G > 64) __syncthreads();
        s = over_row<G, false>(s, parts) / (float)p.D;
        const auto finish = [&](int c, const Raw<T>& d) {
            float f[8];
            unpack_at<T, W>(d, c, p.D, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] += rstd * (g[i] - n[i] * s);
            write(c, f);
        };
        if (N > 0) {
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                const int c = lane + k * G;
                if (c >= chunks) continue;
                if (!kAhead || W != kWhole) {
                    hide(a[k]);
                    hide(b[k]);
                }
                if (!kAhead) load_weight<T, W>(p.weight, p.weight_f32, c, p.D, w[k]);
                take(c, a[k], b[k], w[k], n, g, nullptr);
                finish(c, d[k]);
            }
        } else {
            for (int c = lane; c < chunks; c += G) {
                load_weight<T, W>(p.weight, p.weight_f32, c, p.D, w[0]);
                take(c, raw_at<T, W>(row_of(row), c, p.D),
                     p.grad_y ? raw_at<T, W>(dy_of(row), c, p.D) : no_values<T>(), w[0], n, g, nullptr);
                finish(c, dsum ? raw_at<T, W>(dsum, c, p.D) : no_values<T>());
            }
        }
    }
    if (N == 0 || !partial) return;
    if (G == 64) {
        __shared__ float join[kRows][64 * kHeld * 8];
        for (int k = 0; k < kHeld; ++k)
            for (int i = 0; i < 8; ++i) join[sub][(k * 8 + i) * 64 + lane] = dw[k][i];
        __syncthreads();
        if (sub > 0) return;
        for (int k = 0; k < kHeld; ++k)
            for (int i = 0; i < 8; ++i)
                for (int w = 1; w < kRows; ++w) dw[k][i] += join[w][(k * 8 + i) * 64 + lane];
    }
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
        const int c = lane + k * G;
        if (c >= chunks) continue;
        if (p.add) {
            float old[8];
            load_at<F32, W>(partial, c, p.D, old);
#pragma unroll
            for (int i = 0; i < 8; ++i) dw[k][i] += old[i];
        }
        store_at<F32, W>(partial, c, p.D, dw[k]);
    }
}

// Columns of the partial sums, added up in the order of the workgroups: 32 columns and 32 stretches of rows a
// workgroup, 16 loads at once (5 us for 768 x 640; 11 one at a time).
constexpr int kColumns = 32, kStretches = 32, kAtOnce = 16;
template <typename T>
__global__ __launch_bounds__(kColumns * kStretches) void k_norm_weight(const float* partials, int blocks, int D,
                                                                       typename T::Store* out)
{
    __shared__ float sums[kStretches][kColumns + 1];
    const int column = threadIdx.x % kColumns, stretch = threadIdx.x / kColumns;
    const int at = blockIdx.x * kColumns + column;
    const int each = (blocks + kStretches - 1) / kStretches;
    const int to = min(blocks, (stretch + 1) * each);
    float s = 0.f;
    if (at < D)
        for (int b = stretch * each; b < to; b += kAtOnce) {
            float f[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) f[k] = b + k < to ? partials[(int64_t)(b + k) * D + at] : 0.f;
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) s += f[k];
        }
    sums[stretch][column] = s;
    __syncthreads();
    if (stretch > 0 || at >= D) return;
    for (int k = 1; k < kStretches; ++k) s += sums[k][column];
    T::store(out + at, s);
}

template <int G_, int N_>
struct Shape {
    static constexpr int G = G_, N = N_;
};

// Lanes and chunks of a row, forward: us of fp32 / bf16, dropout 0.1, replayed, first what is taken (a width of both for one type
// alone where the other keeps what follows it). Rows of 640 32,000; 1,101 40,000; 1,500, 2,000 and 2,001 32,000; 2,500 16,000; 2,501
// and 3,001 24,000; 4,096, 5,000 and 5,003 16,000; 6,000 and 6,001 14,000; 7,001 12,000; 8,192 8,000; 9,001 9,000; 12,000 8,000; 16,384
// 6,000.
//    640:    64 x 2 65 / 32, 128 x 1 69 / 42
//    1,101:  64 x 3 138 / 81, 64 x 4 137 / 89, 128 x 2 142 / 99
//    1,500:  64 x 3 153 / 75, 128 x 2 153 / 81
//    2,000:  64 x 4 194 / 99, 128 x 2 204 / 96 (bf16: this); 2,001: 195 / 105 and 205 / 114
//    2,500:  192 x 2 129 / 68, 256 x 2 130 / 94; 2,501: 185 / 108, 64 x 5 195 / 101 (bf16: this), 128 x 3 189 / 112
//    3,001:  192 x 2 223 / 120, 128 x 3 227 / 124, 64 x 6 232 / 137
//    4,096:  256 x 2 192 / 103, 512 x 1 185 / 105; 20,000 of 4,001: 245 / 136, 128 x 4 249 / 144
//    5,000:  256 x 4 233 / 117, 128 x 5 256 / 117, 320 x 2 243 / 117, 640 x 1 228 / 156; 5,003: 233 / 153, 240 / 146 (bf16: this), 233 / 168, 233 / 188
//    6,000:  256 x 4 249 / 119, 256 x 3 263 / 119; 6,001: 245 / 152, 257 / 145 (bf16: this)
//    7,001:  256 x 4 249 / 150, 192 x 6 259 / 219, 128 x 8 260 / 167
//    8,192:  256 x 4 193 / 106, 512 x 2 190 / 104, 1024 x 1 192 / 126
//    9,001:  512 x 3 245 / 169, 768 x 2 248 / 208, 1024 x 2 259 / 218, 384 x 4 287 / 190; 12,000: 283 / 139, 278 / 160, 301 / 167, 304 / 148
//    16,384: 1024 x 2 288 / 150, 512 x 4 305 / 137, chunks read again 319 / 202; 13,001: 254 / 181 and 272 / 197
// Few rows leave most of the chip idle, and each is spread over more lanes (256 rows of bf16): 640: 256 x 1 3.8, 64 x 2 4.5. 2,048: 256
// x 1 4.0, 128 x 2 4.6. 4,096: 512 x 1 4.6, 256 x 2 5.0. 8,192: 512 x 2 6.3, 256 x 4 7.1; 1,024 rows of 640: 5.4 and 4.7, of 4,096: 8.9
// and 8.7.
constexpr int kFewRows = 512;
template <typename F>
void by_shape(int64_t rows, int D, int dtype, F&& f)
{
    const int chunks = (D + 7) / 8;
    const bool half = dtype != LFMMI_F32, odd = D % 8 != 0;
    if (chunks <= 64) f(Shape<64, 1>{});
    else if (rows <= kFewRows && chunks <= 256) f(Shape<256, 1>{});
    else if (rows <= kFewRows && chunks <= 512) f(Shape<512, 1>{});
    else if (rows <= kFewRows && chunks <= 1024) f(Shape<512, 2>{});
    else if (chunks <= 128) f(Shape<64, 2>{});
    else if (chunks <= 192) f(Shape<64, 3>{});
    else if (chunks <= 256 && (!half || odd)) f(Shape<64, 4>{});
    else if (chunks <= 256) f(Shape<128, 2>{});
    else if (chunks <= 320 && half && odd) f(Shape<64, 5>{});
    else if (chunks <= 384) f(Shape<192, 2>{});
    else if (chunks <= 512) f(Shape<256, 2>{});
    else if (chunks <= 640 && half) f(Shape<128, 5>{});
    else if (chunks <= 768 && half) f(Shape<256, 3>{});
    else if (chunks <= 1024) f(Shape<256, 4>{});
    else if (chunks <= 1536) f(Shape<512, 3>{});
    else if (chunks <= 2048) f(Shape<1024, 2>{});
    else f(Shape<1024, 0>{});
}

// ... and backward, with the workgroups that go round the rows, as many as the registers leave place for (the same rows; 500 60,000, 2,048
// 16,000, 2,496 24,000, 4,100 16,000, 8,190 9,000).
//    500:    64 x 1 1,024 127 / 63, 2,048 130 / 74
//    640:    64 x 2 768 84 / 38, 1,024 88 / 44, 128 x 1 2,048 87 / 41
//    1,101:  256 x 1 1,024 181 / 129, 192 x 1 1,024 181 / 130, 128 x 2 1,024 179 / 158
//    2,048:  256 x 1 1,024 128 / 65, 128 x 2 1,024 128 / 67; 2,001: 259 / 146, 255 / 150, 64 x 4 512 253 / 176
//    2,496:  512 x 1 512 222 / 125, 192 x 2 768 224 / 120 (bf16: this), 320 x 1 768 229 / 116; 2,501: 232 / 165, 279 / 144, 267 / 207
//    3,001:  512 x 1 512 277 / 171, 192 x 2 768 319 / 162, 384 x 1 512 278 / 170, 128 x 3 512 273 / 221
//    4,096:  512 x 1 512 243 / 128, 256 x 2 512 240 / 124; 20,000 of 4,001: 308 / 177 and 308 / 181
//    4,100:  640 x 1 256 248 / 198, 512 x 2 256 261 / 224; 5,003: 298 / 230 and 295 / 240
//    6,000:  512 x 2 256 316 / 156, 256 x 3 512 323 / 160, 384 x 2 256 314 / 190; 6,001: 318 / 209, 323 / 192 (bf16: this), 310 / 246
//    8,192:  512 x 2 256 256 / 126, 512 254 / 134, 1024 x 1 250 / 126; 8,190: 285 / 159, 1024 x 1 282 / 138; 7,001: 323 / 217, 319 / 200 (bf16: this)
//    9,001:  768 x 2 256 365 / 184, 512 x 3 256 327 / 199, 512 x 4 256 567 / 320, 1024 x 2 624 / 388; 12,000: 376 / 174, 376 / 173, 409 / 224, 403 / 292
//    16,384: 512 x 4 256 412 / 215, 512 blocks 411 / 233, 768 x 3 546 / 307, 1024 x 2 419 / 283, chunks read again 536 / 344
template <int G_, int N_, int Blocks_>
struct Rounds : Shape<G_, N_> {
    static constexpr int kBlocks = Blocks_;
};
template <typename F>
void by_rounds(int D, int dtype, F&& f)
{
    const int chunks = (D + 7) / 8;
    const bool half = dtype != LFMMI_F32, odd = D % 8 != 0;
    if (chunks <= 64) f(Rounds<64, 1, 1024>{});
    else if (chunks <= 128) f(Rounds<64, 2, 768>{});
    else if (chunks <= 256) f(Rounds<256, 1, 1024>{});
    else if (chunks <= 384 && half) f(Rounds<192, 2, 768>{});
    else if (chunks <= 512) f(Rounds<512, 1, 512>{});
    else if (chunks <= 640) f(Rounds<640, 1, 256>{});
    else if (chunks <= 768 && half && odd) f(Rounds<256, 3, 512>{});
    else if (chunks > 768 && chunks <= 1024 && half && odd) f(Rounds<1024, 1, 256>{});
    else if (chunks <= 1024) f(Rounds<512, 2, 256>{});
    else if (chunks <= 1536) f(Rounds<768, 2, 256>{});
    else if (chunks <= 2048) f(Rounds<512, 4, 256>{});
    else f(Rounds<1024, 0, 256>{});
}

}  // namespace

hipError_t launch_dropout(const DropoutParams& p, int dtype, hipStream_t stream)
{
    const int64_t chunks = ((int64_t)p.D + 7) / 8;
    int lanes_log2 = 0;
    while ((1 << lanes_log2) < kThreads && (1 << lanes_log2) < chunks) ++lanes_log2;
    const int rows = kThreads >> lanes_log2;
    const int64_t piece = (int64_t)kDropoutChunks << lanes_log2;
    const int64_t pieces = (chunks + piece - 1) / piece, units = ((int64_t)p.R + rows - 1) / rows * pieces;
    if (units > UINT32_MAX - (1 << 20)) return hipErrorInvalidValue;
    const int grid = (int)std::min<int64_t>(units, 1 << 20);
    by_type(dtype, [&](auto t) {
        by_width<true>(p.D, [&](auto whole) {
            k_dropout<decltype(t), decltype(whole)::value>
                <<<grid, kThreads, 0, stream>>>(p, lanes_log2, (uint32_t)pieces, (uint32_t)units);
        });
    });
    return hipGetLastError();
}

hipError_t launch_norm(const NormParams& p, const SeqLengths& lens, int dtype, hipStream_t stream)
{
    const int64_t rows = (int64_t)p.B * p.T;
    by_type(dtype, [&](auto t) {
        by_shape(rows, p.D, dtype, [&](auto s) {
            constexpr int G = decltype(s)::G, N = decltype(s)::N, kRows = threads_of(G) / G;
            const int grid = (int)std::min<int64_t>((rows + kRows - 1) / kRows, 1 << 20);
            by_width<G == 64 && N == 1>(p.D, [&](auto whole) {
                k_norm<decltype(t), decltype(whole)::value, G, N><<<grid, threads_of(G), 0, stream>>>(p, lens);
            });
        });
    });
    return hipGetLastError();
}

int norm_blocks(int64_t rows, int D, int dtype)
{
    int blocks = 0;
    by_rounds(D, dtype, [&](auto s) {
        constexpr int G = decltype(s)::G, kRows = threads_of(G) / G;
        blocks = (int)std::min<int64_t>((rows + kRows - 1) / kRows, decltype(s)::kBlocks);
    });
    return blocks;
}

hipError_t launch_norm_grad(const NormGradParams& p, const SeqLengths& lens, int dtype, hipStream_t stream)
{
    by_type(dtype, [&](auto t) {
        by_rounds(p.D, dtype, [&](auto s) {
            constexpr int G = decltype(s)::G, N = decltype(s)::N;
            by_width<G == 64 && N == 1>(p.D, [&](auto whole) {
                k_norm_grad<decltype(t), decltype(whole)::value, G, N><<<p.blocks, threads_of(G), 0, stream>>>(p, lens);
            });
        });
    });
    return hipGetLastError();
}

hipError_t launch_norm_weight(const float* partials, int blocks, int D, void* grad_weight, int dtype,
                              hipStream_t stream)
{
    by_type(dtype, [&](auto t) {
        using T = decltype(t);
        k_norm_weight<T><<<(D + kColumns - 1) / kColumns, kColumns * kStretches, 0, stream>>>(
            partials, blocks, D, static_cast<typename T::Store*>(grad_weight));
    });
    return hipGetLastError();
}

}  // namespace lfmmi
