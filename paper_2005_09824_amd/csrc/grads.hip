// The norm of many gradient tensors taken together, and gradients scaled to a norm.
#include <hip/hip_runtime.h>

#include "../../include/lfmmi.h"
#include "operators.h"
#include "vec16.h"

namespace lfmmi {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// The sum over a workgroup, the same bits in every thread.
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double parts[kWaves];
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.;
    for (int w = 0; w < kWaves; ++w) v += parts[w];
    return v;
}

// The last tensor whose first unit is not after `unit`.
__device__ __forceinline__ int tensor_of(const GradList& l, int unit)
{
    int lo = 0, hi = l.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (l.first[mid] <= unit) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The units of a workgroup: a stretch of them one after the other, so that the tensor is
// looked up once and then followed.
struct Stretch {
    int from, to;
};
__device__ __forceinline__ Stretch stretch_of(const GradList& l)
{
    const int64_t units = l.first[kGradTensors];
    return {(int)(units * blockIdx.x / gridDim.x), (int)(units * (blockIdx.x + 1) / gridDim.x)};
}

// Sums of squares in fp64: a float's square overflows a float from 2^64 on, and the sum of 1e9 of
// them keeps 9 digits more than it is rounded to.
template <typename D>
__device__ __forceinline__ double squares(const void* at, int n)
{
    using Store = typename D::Store;
    constexpr int kLoads = kGradUnit / kThreads / D::kVec;
    const Store* x = static_cast<const Store*>(at);
    double s[4] = {0., 0., 0., 0.};
    if (n == kGradUnit) {
        uint4 r[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) r[k] = load16(x + (threadIdx.x + k * kThreads) * D::kVec);
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            float f[D::kVec];
            D::unpack(r[k], f);
#pragma unroll
            for (int i = 0; i < D::kVec; ++i) s[i & 3] += (double)f[i] * (double)f[i];
        }
    } else {
        const int full = n / D::kVec;
        for (int q = threadIdx.x; q < full; q += kThreads) {
            float f[D::kVec];
            D::unpack(load16(x + q * D::kVec), f);
#pragma unroll
            for (int i = 0; i < D::kVec; ++i) s[i & 3] += (double)f[i] * (double)f[i];
        }
        for (int i = full * D::kVec + threadIdx.x; i < n; i += kThreads) {
            const double v = D::load(x + i);
            s[0] += v * v;
        }
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
}

__global__ __launch_bounds__(kThreads) void k_grad_squares(GradList l, double* partials)
{
    double sum = 0.;
    const Stretch st = stretch_of(l);
    for (int u = st.from, i = tensor_of(l, u); u < st.to; ++u) {
        while (l.first[i + 1] <= u) ++i;
        const int dtype = (int)(l.count[i] & 3);
        const int64_t from = (int64_t)(u - l.first[i]) * kGradUnit, left = (l.count[i] >> 2) - from;
        const int n = left < kGradUnit ? (int)left : kGradUnit;
        if (dtype == LFMMI_F32) sum += squares<F32>(static_cast<const float*>(l.in[i]) + from, n);
        else if (dtype == LFMMI_BF16) sum += squares<Bf16>(static_cast<const uint16_t*>(l.in[i]) + from, n);
        else sum += squares<F16>(static_cast<const _Float16*>(l.in[i]) + from, n);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) partials[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kThreads) void k_grad_norm(const double* partials, int n, float max_norm,
                                                        float* norm, float* factor)
{
    double sum = 0.;
    for (int i = threadIdx.x; i < n; i += kThreads) sum += partials[i];
    sum = block_sum(sum);
    if (threadIdx.x) return;
    const double root = sqrt(sum);
    const float rounded = (float)root;
    *norm = rounded;
    if (max_norm < 0.f) return;
    // a norm that is not finite: every gradient becomes 0
    if (!(rounded < INFINITY)) *factor = 0.f;
    else *factor = root > (double)max_norm ? (float)((double)max_norm / root) : 1.f;
}

// (a factor of 0 makes a NaN 0 too)
template <typename D>
__device__ __forceinline__ void scale(const void* at, void* to, int n, float factor)
{
    using Store = typename D::Store;
    constexpr int kLoads = kGradUnit / kThreads / D::kVec;
    const Store* x = static_cast<const Store*>(at);
    Store* y = static_cast<Store*>(to);
    if (n == kGradUnit) {
        uint4 r[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) r[k] = load16(x + (threadIdx.x + k * kThreads) * D::kVec);
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            float f[D::kVec];
            D::unpack(r[k], f);
#pragma unroll
            for (int i = 0; i < D::kVec; ++i) f[i] = factor == 0.f ? 0.f : f[i] * factor;
            store16(y + (threadIdx.x + k * kThreads) * D::kVec, D::pack(f));
        }
    } else {
        const int full = n / D::kVec;
        for (int q = threadIdx.x; q < full; q += kThreads) {
            float f[D::kVec];
            D::unpack(load16(x + q * D::kVec), f);
#pragma unroll
            for (int i = 0; i < D::kVec; ++i) f[i] = factor == 0.f ? 0.f : f[i] * factor;
            store16(y + q * D::kVec, D::pack(f));
        }
        for (int i = full * D::kVec + threadIdx.x; i < n; i += kThreads)
            D::store(y + i, factor == 0.f ? 0.f : D::load(x + i) * factor);
    }
}

// The units are gone through from the last to the first: what k_grad_squares read last is still in
// the 256 MB cache.
__global__ __launch_bounds__(kThreads) void k_grad_scale(GradList l, const float* factor)
{
    const float f = *factor;
    const Stretch st = stretch_of(l);
    for (int u = st.to - 1, i = tensor_of(l, u); u >= st.from; --u) {
        while (l.first[i] > u) --i;
        if (f == 1.f && l.in[i] == l.out[i]) continue;  // in place and nothing to scale
        const int dtype = (int)(l.count[i] & 3);
        const int64_t from = (int64_t)(u - l.first[i]) * kGradUnit, left = (l.count[i] >> 2) - from;
        const int n = left < kGradUnit ? (int)left : kGradUnit;
        const int64_t at = from * (dtype == LFMMI_F32 ? 4 : 2);
        const void* in = static_cast<const char*>(l.in[i]) + at;
        void* out = static_cast<char*>(l.out[i]) + at;
        if (dtype == LFMMI_F32) scale<F32>(in, out, n, f);
        else if (dtype == LFMMI_BF16) scale<Bf16>(in, out, n, f);
        else scale<F16>(in, out, n, f);
    }
}

}  // namespace

int grad_blocks(const GradList& l)
{
    const int units = l.first[kGradTensors];
    return units < kGradBlocks ? units : kGradBlocks;
}

hipError_t launch_grad_squares(const GradList& l, double* partials, hipStream_t stream)
{
    k_grad_squares<<<grad_blocks(l), kThreads, 0, stream>>>(l, partials);
    return hipGetLastError();
}

hipError_t launch_grad_norm(const double* partials, int n, float max_norm, float* norm,
                            float* factor, hipStream_t stream)
{
    k_grad_norm<<<1, kThreads, 0, stream>>>(partials, n, max_norm, norm, factor);
    return hipGetLastError();
}

hipError_t launch_grad_scale(const GradList& l, const float* factor, hipStream_t stream)
{
    k_grad_scale<<<grad_blocks(l), kThreads, 0, stream>>>(l, factor);
    return hipGetLastError();
}

}  // namespace lfmmi
