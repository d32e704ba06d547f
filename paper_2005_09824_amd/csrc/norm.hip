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
constexpr float kLeastScale = 1.17549435e-38f;  // 2^-126: its inverse is finite

constexpr int threads_of(int lanes) { return lanes > kThreads ? lanes : kThreads; }

// ---- dropout alone

constexpr int kDropoutChunks = 4;  // of eight values, that a lane takes of a row

template <typename T>
__global__ __launch_bounds__(kThreads) void k_dropout(DropoutParams p, int lanes_log2, uint32_t pieces, uint32_t units)
{
    using Store = typename T::Store;
    const Dropping drop(p.draw);
    const int lanes = 1 << lanes_log2, lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> lanes_log2;
    const int rows = kThreads >> lanes_log2;
    for (uint32_t u = blockIdx.x; u < units; u += gridDim.x) {
        const uint32_t group = u / pieces;
        const int64_t row = (int64_t)group * rows + sub;
        if (row >= p.R) continue;
        const Store* x = static_cast<const Store*>(p.x) + row * p.stride_x;
        Store* y = static_cast<Store*>(p.y) + row * p.stride_y;
        const int64_t first = (int64_t)(u - group * pieces) * kDropoutChunks * lanes + lane;
        float f[kDropoutChunks][8];
#pragma unroll
        for (int k = 0; k < kDropoutChunks; ++k) {
            const int64_t c = first + k * lanes;
            if (c * 8 < p.D) load8<T>(x + c * 8, (int)min((int64_t)8, p.D - c * 8), f[k]);
        }
#pragma unroll
        for (int k = 0; k < kDropoutChunks; ++k) {
            const int64_t c = first + k * lanes;
            if (c * 8 >= p.D) continue;
            if (drop.threshold > 0) drop.apply((uint32_t)row, (uint32_t)c, f[k]);
            store8<T>(y + c * 8, (int)min((int64_t)8, p.D - c * 8), f[k]);
        }
    }
}

// ---- norms

// The sum, or the largest, over the G lanes that take a row.
template <int G>
struct Join {
    float parts[2][G / 64];
};
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

template <typename T>
__device__ __forceinline__ void load_weight(const void* w, bool f32, int c, int left, float* f)
{
    if (!w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = 1.f;
    } else if (f32) {
        load8<F32>(static_cast<const float*>(w) + c * 8, left, f);
    } else {
        load8<T>(static_cast<const typename T::Store*>(w) + c * 8, left, f);
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
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) q[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
}

// A value as it is kept in the type.
template <typename T>
__device__ __forceinline__ float rounded(float v)
{
    if (T::kVec == 4) return v;
    typename T::Store s;
    T::store(&s, v);
    return T::load(&s);
}

// Bits of |y| as whole numbers: the largest of them is a NaN's, if there is one.
__device__ __forceinline__ uint32_t magnitude(float y) { return __float_as_uint(y) & 0x7fffffffu; }

// G lanes take a row, N chunks of eight values each, which stay in registers; N == 0: any number of
// chunks, read again for each pass over the row.
template <typename T, int G, int N>
__global__ __launch_bounds__(threads_of(G)) void k_norm(NormParams p, SeqLengths lens)
{
    using Store = typename T::Store;
    constexpr int kRows = threads_of(G) / G;
    constexpr int kHeld = N > 0 ? N : 1;
    __shared__ float parts[2][G / 64];
    const Dropping drop(p.draw);
    const int lane = threadIdx.x % G, chunks = (p.D + 7) / 8;
    const uint32_t rows = (uint32_t)p.B * (uint32_t)p.T;
    for (uint32_t row = blockIdx.x * kRows + threadIdx.x / G; row < rows; row += gridDim.x * kRows) {
        const Store* x = static_cast<const Store*>(p.x) + offset_of(row, p.T, p.x_stride_b, p.x_stride_t);
        const Store* res = p.residual
            ? static_cast<const Store*>(p.residual) + offset_of(row, p.T, p.r_stride_b, p.r_stride_t) : nullptr;
        const int64_t at = (int64_t)row * p.D;
        Store* sum = p.sum ? static_cast<Store*>(p.sum) + at : nullptr;
        Store* y = p.y ? static_cast<Store*>(p.y) + at : nullptr;
        uint8_t* q = p.q ? p.q + at : nullptr;
        float h[kHeld][8];
        const auto left_of = [&](int c) { return p.D - c * 8; };
        if (!inside(lens, row, p.T)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) h[0][i] = 0.f;
            for (int c = lane; c < chunks; c += G) {
                if (sum) store8<T>(sum + c * 8, left_of(c), h[0]);
                if (y) store8<T>(y + c * 8, left_of(c), h[0]);
                if (q) store_bytes(q + c * 8, left_of(c), h[0]);
            }
            if (lane == 0) {
                if (p.rstd) p.rstd[row] = 0.f;
                if (p.q_scale) p.q_scale[row] = 0.f;
            }
            continue;
        }
        const auto added = [&](int c, float* f) {
            float r[8];
            load8<T>(x + c * 8, left_of(c), f);
            if (res) load8<T>(res + c * 8, left_of(c), r);
            if (drop.threshold > 0) drop.apply((uint32_t)(p.row + row), (uint32_t)c, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = rounded<T>(res ? f[i] + r[i] : f[i]);
        };
        float s = 0.f;
        if (N > 0) {
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                const int c = lane + k * G;
                if (c < chunks) {
                    added(c, h[k]);
                    if (sum) store8<T>(sum + c * 8, left_of(c), h[k]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[k][i] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) s = fmaf(h[k][i], h[k][i], s);
            }
        } else {
            for (int c = lane; c < chunks; c += G) {
                added(c, h[0]);
                if (sum) store8<T>(sum + c * 8, left_of(c), h[0]);
#pragma unroll
                for (int i = 0; i < 8; ++i) s = fmaf(h[0][i], h[0][i], s);
            }
        }
        if (G > 64) __syncthreads();  // (the row before has read `parts`)
        s = over_row<G, false>(s, parts[0]);
        float rstd = 1.f / sqrtf(s / (float)p.D + p.eps);
        if (__builtin_expect(!(s < INFINITY), 0)) {  // squares beyond fp32, unless there is an infinity or a NaN: taken again of smaller values
            s = 0.f;
            if (N > 0) {
#pragma unroll
                for (int k = 0; k < kHeld; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) s = fmaf(h[k][i] * kSmaller, h[k][i] * kSmaller, s);
            } else {
                for (int c = lane; c < chunks; c += G) {
                    load8<T>(sum ? sum + c * 8 : x + c * 8, left_of(c), h[0]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) s = fmaf(h[0][i] * kSmaller, h[0][i] * kSmaller, s);
                }
            }
            s = over_row<G, false>(s, parts[1]);
            rstd = kSmaller / sqrtf(s / (float)p.D);
            if (G > 64) __syncthreads();
        }
        if (p.rstd && lane == 0) p.rstd[row] = rstd;
        // (what a lane has written itself is read again: from `sum`, or from x where nothing was added)
        const auto scaled = [&](int c, int k, float* f) {
            float w[8];
            load_weight<T>(p.weight, p.weight_f32, c, left_of(c), w);
            if (N == 0) load8<T>(sum ? sum + c * 8 : x + c * 8, left_of(c), h[0]);
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
                if (y) store8<T>(y + c * 8, left_of(c), f);
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
                if (y) store8<T>(y + c * 8, left_of(c), f);
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
        const float inverse = 1.f / scale;
        if (p.q_scale && lane == 0) p.q_scale[row] = scale;
        if (N > 0) {
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                const int c = lane + k * G;
                if (c >= chunks) continue;
#pragma unroll
                for (int i = 0; i < 8; ++i) h[k][i] *= inverse;
                store_bytes(q + c * 8, left_of(c), h[k]);
            }
        } else {
            for (int c = lane; c < chunks; c += G) {
                float f[8];
                scaled(c, 0, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= inverse;
                store_bytes(q + c * 8, left_of(c), f);
            }
        }
    }
}

// The same lanes and chunks; a workgroup adds its rows' share of the weight's gradient up, and leaves it as a
// row of partial sums.
template <typename T, int G, int N>
__global__ __launch_bounds__(threads_of(G)) void k_norm_grad(NormGradParams p, SeqLengths lens)
{
    using Store = typename T::Store;
    constexpr int kRows = threads_of(G) / G;
    constexpr int kHeld = N > 0 ? N : 1;
    __shared__ float parts[G / 64];
    const Dropping drop(p.draw);
    const int lane = threadIdx.x % G, sub = threadIdx.x / G, chunks = (p.D + 7) / 8;
    const uint32_t rows = (uint32_t)p.B * (uint32_t)p.T;
    float dw[kHeld][8];
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[k][i] = 0.f;
    float* partial = p.partials ? p.partials + (int64_t)blockIdx.x * p.D : nullptr;
    if (N == 0 && partial && !p.add)
        for (int c = lane; c < chunks; c += G) store8<F32>(partial + c * 8, p.D - c * 8, dw[0]);
    for (uint32_t row = blockIdx.x * kRows + sub; row < rows; row += gridDim.x * kRows) {
        const int64_t at = (int64_t)row * p.D;
        const Store* hr = static_cast<const Store*>(p.h) + offset_of(row, p.T, p.stride_b, p.stride_t);
        const Store* dy = p.grad_y ? static_cast<const Store*>(p.grad_y) + at : nullptr;
        const Store* dsum = p.grad_sum ? static_cast<const Store*>(p.grad_sum) + at : nullptr;
        Store* dx = p.grad_x ? static_cast<Store*>(p.grad_x) + at : nullptr;
        Store* dres = p.grad_residual ? static_cast<Store*>(p.grad_residual) + at : nullptr;
        const auto left_of = [&](int c) { return p.D - c * 8; };
        const auto write = [&](int c, float* f) {
            if (dres) store8<T>(dres + c * 8, left_of(c), f);
            if (dx) {
                if (drop.threshold > 0) drop.apply((uint32_t)(p.row + row), (uint32_t)c, f);
                store8<T>(dx + c * 8, left_of(c), f);
            }
        };
        if (!inside(lens, row, p.T)) {
            float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (int c = lane; c < chunks; c += G) {
                if (dres) store8<T>(dres + c * 8, left_of(c), zero);
                if (dx) store8<T>(dx + c * 8, left_of(c), zero);
            }
            continue;
        }
        const float rstd = p.rstd[row];
        float h[kHeld][8], g[kHeld][8];
        // h and w dy of a chunk; the weight's gradient on the way
        const auto take = [&](int c, float* h, float* g, float* dw) {
            float w[8];
            load8<T>(hr + c * 8, left_of(c), h);
            if (!dy) {
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = 0.f;
                return;
            }
            load8<T>(dy + c * 8, left_of(c), g);
            load_weight<T>(p.weight, p.weight_f32, c, left_of(c), w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[i] *= rstd;
                if (dw) dw[i] = fmaf(g[i], h[i], dw[i]);
                g[i] *= w[i];
            }
        };
        float s = 0.f;
        if (N > 0) {
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                const int c = lane + k * G;
                if (c >= chunks) continue;
                take(c, h[k], g[k], dw[k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) s = fmaf(g[k][i], h[k][i], s);
            }
        } else {
            for (int c = lane; c < chunks; c += G) {
                float add[8];
                if (partial) load8<F32>(partial + c * 8, left_of(c), add);
                take(c, h[0], g[0], partial ? add : nullptr);
                if (partial) store8<F32>(partial + c * 8, left_of(c), add);
#pragma unroll
                for (int i = 0; i < 8; ++i) s = fmaf(g[0][i], h[0][i], s);
            }
        }
        if (G > 64) __syncthreads();
        s = over_row<G, false>(s, parts) / (float)p.D;
        const auto finish = [&](int c, const float* h, const float* g) {
            float f[8];
            if (dsum) load8<T>(dsum + c * 8, left_of(c), f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = rstd * (g[i] - h[i] * s);
                f[i] = dsum ? f[i] + d : d;
            }
            write(c, f);
        };
        if (N > 0) {
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                const int c = lane + k * G;
                if (c < chunks) finish(c, h[k], g[k]);
            }
        } else {
            for (int c = lane; c < chunks; c += G) {
                take(c, h[0], g[0], nullptr);
                finish(c, h[0], g[0]);
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
            load8<F32>(partial + c * 8, p.D - c * 8, old);
#pragma unroll
            for (int i = 0; i < 8; ++i) dw[k][i] += old[i];
        }
        store8<F32>(partial + c * 8, p.D - c * 8, dw[k]);
    }
}

// Columns of the partial sums, added up in the order of the workgroups: 32 columns and 32 stretches of rows a
// workgroup.
constexpr int kColumns = 32, kStretches = 32;
template <typename T>
__global__ __launch_bounds__(kColumns * kStretches) void k_norm_weight(const float* partials, int blocks, int D,
                                                                       typename T::Store* out)
{
    __shared__ float sums[kStretches][kColumns + 1];
    const int column = threadIdx.x % kColumns, stretch = threadIdx.x / kColumns;
    const int at = blockIdx.x * kColumns + column;
    const int each = (blocks + kStretches - 1) / kStretches;
    float s = 0.f;
    if (at < D)
        for (int b = stretch * each; b < min(blocks, (stretch + 1) * each); ++b) s += partials[(int64_t)b * D + at];
    sums[stretch][column] = s;
    __syncthreads();
    if (stretch > 0 || at >= D) return;
    for (int k = 1; k < kStretches; ++k) s += sums[k][column];
    T::store(out + at, s);
}

template <typename F>
void by_type(int dtype, F&& f)
{
    if (dtype == LFMMI_F32) f(F32{});
    else if (dtype == LFMMI_BF16) f(Bf16{});
    else f(F16{});
}

template <int G_, int N_>
struct Shape {
    static constexpr int G = G_, N = N_;
};

// Lanes and chunks of a row.
template <typename F>
void by_shape(int D, F&& f)
{
    const int chunks = (D + 7) / 8;
    if (chunks <= 64) f(Shape<64, 1>{});
    else if (chunks <= 128) f(Shape<64, 2>{});
    else if (chunks <= 256) f(Shape<64, 4>{});
    else if (chunks <= 512) f(Shape<256, 2>{});
    else if (chunks <= 1024) f(Shape<256, 4>{});
    else if (chunks <= 2048) f(Shape<1024, 2>{});
    else f(Shape<1024, 0>{});
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
        k_dropout<decltype(t)><<<grid, kThreads, 0, stream>>>(p, lanes_log2, (uint32_t)pieces, (uint32_t)units);
    });
    return hipGetLastError();
}

hipError_t launch_norm(const NormParams& p, const SeqLengths& lens, int dtype, hipStream_t stream)
{
    const int64_t rows = (int64_t)p.B * p.T;
    by_type(dtype, [&](auto t) {
        by_shape(p.D, [&](auto s) {
            constexpr int G = decltype(s)::G, N = decltype(s)::N, kRows = threads_of(G) / G;
            const int grid = (int)std::min<int64_t>((rows + kRows - 1) / kRows, 1 << 20);
            k_norm<decltype(t), G, N><<<grid, threads_of(G), 0, stream>>>(p, lens);
        });
    });
    return hipGetLastError();
}

int norm_blocks(int64_t rows, int D)
{
    int blocks = 0;
    by_shape(D, [&](auto s) {
        constexpr int G = decltype(s)::G, kRows = threads_of(G) / G;
        blocks = (int)std::min<int64_t>((rows + kRows - 1) / kRows, G == 1024 ? 512 : kNormBlocks);
    });
    return blocks;
}

hipError_t launch_norm_grad(const NormGradParams& p, const SeqLengths& lens, int dtype, hipStream_t stream)
{
    by_type(dtype, [&](auto t) {
        by_shape(p.D, [&](auto s) {
            constexpr int G = decltype(s)::G, N = decltype(s)::N;
            k_norm_grad<decltype(t), G, N><<<p.blocks, threads_of(G), 0, stream>>>(p, lens);
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
