// The norm of many gradient tensors taken together, and gradients scaled to a norm.
#include <hip/hip_runtime.h>

#include "../../include/lfmmi.h"
#include "operators.h"

namespace lfmmi {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

__device__ __forceinline__ float load(const void* p, int64_t i, int dtype)
{
    if (dtype == LFMMI_F32) return static_cast<const float*>(p)[i];
    if (dtype == LFMMI_BF16)
        return __uint_as_float((uint32_t) static_cast<const uint16_t*>(p)[i] << 16);
    return (float)static_cast<const _Float16*>(p)[i];
}

// (to nearest, ties to even)
__device__ __forceinline__ void store(void* p, int64_t i, int dtype, float v)
{
    if (dtype == LFMMI_F32)
        static_cast<float*>(p)[i] = v;
    else if (dtype == LFMMI_BF16)
        static_cast<uint16_t*>(p)[i] = __builtin_bit_cast(uint16_t, (__bf16)v);
    else
        static_cast<_Float16*>(p)[i] = (_Float16)v;
}

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

__global__ __launch_bounds__(kThreads) void k_grad_squares(GradList l, double* partials)
{
    double sum = 0.;
    const int units = l.first[kGradTensors];
    for (int u = blockIdx.x; u < units; u += gridDim.x) {
        const int i = tensor_of(l, u);
        const int dtype = (int)(l.count[i] & 3);
        const int64_t count = l.count[i] >> 2;
        const int64_t from = (int64_t)(u - l.first[i]) * kGradUnit;
        const int64_t to = from + kGradUnit < count ? from + kGradUnit : count;
        for (int64_t k = from + threadIdx.x; k < to; k += kThreads) {
            const double v = load(l.in[i], k, dtype);
            sum += v * v;
        }
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

__global__ __launch_bounds__(kThreads) void k_grad_scale(GradList l, const float* factor)
{
    const float f = *factor;
    const int units = l.first[kGradTensors];
    for (int u = blockIdx.x; u < units; u += gridDim.x) {
        const int i = tensor_of(l, u);
        if (f == 1.f && l.in[i] == l.out[i]) continue;  // in place and nothing to scale
        const int dtype = (int)(l.count[i] & 3);
        const int64_t count = l.count[i] >> 2;
        const int64_t from = (int64_t)(u - l.first[i]) * kGradUnit;
        const int64_t to = from + kGradUnit < count ? from + kGradUnit : count;
        for (int64_t k = from + threadIdx.x; k < to; k += kThreads)
            store(l.out[i], k, dtype, f == 0.f ? 0.f : load(l.in[i], k, dtype) * f);
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
