// The norm of many gradient tensors taken together, and gradients scaled to a norm.
#include <hip/hip_runtime.h>

#include <algorithm>

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

// The tensors of a call: in the kernel's arguments, or for more of them than those hold in the
// workspace.
struct Listed {
    const GradList& l;
    __device__ const void* in(int i) const { return l.in[i]; }
    __device__ void* out(int i) const { return l.out[i]; }
    __device__ int64_t count(int i) const { return l.count[i]; }
    __device__ int first(int i) const { return l.first[i]; }
};
// Values between the address that kGradAlign divides and a tensor.
__device__ __forceinline__ int values_before(const void* in, int size)
{
    return (int)((uintptr_t)in % kGradAlign) / size;
}
struct Placed {
    const GradPlaces& l;
    __device__ const void* in(int i) const { return l.in[i]; }
    __device__ void* out(int i) const { return const_cast<void*>(l.in[i]); }
    __device__ int64_t count(int i) const
    {
        const int dtype = l.rest[i] & 3, over = l.rest[i] >> 2;
        const int before = values_before(l.in[i], dtype == LFMMI_F32 ? 4 : 2);
        return ((int64_t)(l.first[i + 1] - l.first[i]) * kGradUnit - before - over) << 2 | dtype;
    }
    __device__ int first(int i) const { return l.first[i]; }
};
// (no kernel that reads the table writes it: constant memory, which a wave reads once for its lanes)
template <typename V>
__device__ __forceinline__ V constant(const V* p, int i)
{
    return ((const __attribute__((address_space(4))) V*)(uintptr_t)p)[i];
}
struct Tabled {
    const GradTable& t;
    __device__ const void* in(int i) const { return constant(t.in, i); }
    __device__ void* out(int i) const { return constant(t.out, i); }
    __device__ int64_t count(int i) const { return constant(t.count, i); }
    __device__ int first(int i) const { return constant(t.first, i); }
};
template <typename L>
struct Tensors {
    L list;
    int n;
};
__device__ __forceinline__ Tensors<Listed> tensors(const GradList& l, int n) { return {{l}, n}; }
__device__ __forceinline__ Tensors<Placed> tensors(const GradPlaces& l, int n) { return {{l}, n}; }
__device__ __forceinline__ Tensors<Tabled> tensors(const GradTable& t, int n) { return {{t}, n}; }

// The last tensor whose first unit is not after `unit`.
template <typename L>
__device__ __forceinline__ int tensor_of(const L& l, int n, int unit)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (l.first(mid) <= unit) lo = mid;
        else hi = mid;
    }
    return lo;
}

// A unit of a tensor: its values from..to - 1 belong to the tensor. Units are counted from the last
// address before the tensor that kGradAlign divides, so that whole ones are aligned: 16-byte loads at
// odd multiples of 2 take 30 % longer, a wave's at 16 bytes off a line 15 %.
struct Unit {
    const char* in;
    char* out;
    int from, to, dtype;
};
template <typename L>
__device__ __forceinline__ Unit unit_of(const L& l, int u)
{
    const int i = tensor_of(l.list, l.n, u);
    const char* in = static_cast<const char*>(l.list.in(i));
    const int64_t packed = l.list.count(i), count = packed >> 2;
    const int dtype = (int)(packed & 3), size = dtype == LFMMI_F32 ? 4 : 2;
    const int before = values_before(in, size);
    const int64_t at = (int64_t)(u - l.list.first(i)) * kGradUnit - before, left = count - at;
    return {in + at * size, static_cast<char*>(l.list.out(i)) + at * size, at < 0 ? before : 0,
            left < kGradUnit ? (int)left : kGradUnit, dtype};
}

// Calls each(k, q) for a thread's chunks q of a unit that are the tensor's as a whole, and one(i) for single
// values at either end. The loads of a thread are all on their way before one is waited for.
template <typename D, typename One>
__device__ __forceinline__ void ends_of(const Unit& u, One&& one)
{
    const int whole = (u.from + D::kVec - 1) / D::kVec * D::kVec, rest = u.to / D::kVec * D::kVec;
    const int head = u.from + threadIdx.x, tail = max(whole, rest) + threadIdx.x;
    if (head < min(whole, u.to)) one(head);
    if (tail < u.to) one(tail);
}
template <typename D>
constexpr int kUnitLoads = kGradUnit / kThreads / D::kVec;
template <typename D>
__device__ __forceinline__ bool has(const Unit& u, int q) { return q * D::kVec >= u.from && (q + 1) * D::kVec <= u.to; }
template <typename D>
__device__ __forceinline__ void load_unit(const Unit& u, bool once, uint4* r)
{
    const typename D::Store* x = reinterpret_cast<const typename D::Store*>(u.in);
    if (u.to - u.from < kGradUnit) {
#pragma unroll
        for (int k = 0; k < kUnitLoads<D>; ++k) {
            const int q = threadIdx.x + k * kThreads;
            r[k] = make_uint4(0, 0, 0, 0);
            if (has<D>(u, q)) r[k] = load16(x + q * D::kVec);
        }
    } else if (once) {
#pragma unroll
        for (int k = 0; k < kUnitLoads<D>; ++k) r[k] = load16_once(x + (threadIdx.x + k * kThreads) * D::kVec);
    } else {
#pragma unroll
        for (int k = 0; k < kUnitLoads<D>; ++k) r[k] = load16(x + (threadIdx.x + k * kThreads) * D::kVec);
    }
}

// Sums of squares in fp64: a float's square overflows a float from 2^64 on, and the sum of 1e9 of
// them keeps 9 digits more than it is rounded to. A conversion to fp64 takes the time of some 12 other
// operations (of bf16 4.1 TB/s went through it): a float's exponent and fraction are put in their
// places in a double instead, which makes it |x| 2^-896, of 0 and denormals too, and scaled
// back. Infinities and NaN become 2^128 or more; where a sum says that there may be one
// `Exact` adds up again.
template <bool Exact>
__device__ __forceinline__ void add_square(double& s, float x)
{
    double v = x;
    if (!Exact) {
        const uint32_t w = __float_as_uint(x);
        v = __hiloint2double((int)((w & 0x7fffffffu) >> 3), (int)(w << 29)) * 0x1p896;
    }
    s = fma(v, v, s);
}

template <typename D, bool Exact>
__device__ __forceinline__ double squares(const Unit& u, bool once)
{
    double s[4] = {0., 0., 0., 0.};
    uint4 r[kUnitLoads<D>];
    load_unit<D>(u, once, r);
#pragma unroll
    for (int k = 0; k < kUnitLoads<D>; ++k) {
        float f[D::kVec];
        D::unpack(r[k], f);
#pragma unroll
        for (int i = 0; i < D::kVec; ++i) add_square<Exact>(s[i & 3], f[i]);
    }
    if (u.to - u.from < kGradUnit)
        ends_of<D>(u, [&](int i) {
            add_square<Exact>(s[0], D::load(reinterpret_cast<const typename D::Store*>(u.in) + i));
        });
    return (s[0] + s[1]) + (s[2] + s[3]);
}

template <bool Exact, typename L>
__device__ __forceinline__ double sum_units(const L& l, const GradCall& c)
{
    double sum = 0.;
    // (what the pass that scales, from the last unit to the first, finds in the cache again is left there)
    const int kept = c.units - (int)((int64_t)c.units * c.keep >> 8);
    for (int64_t at = blockIdx.x; at < c.units; at += gridDim.x) {
        const Unit u = unit_of(l, (int)at);
        const bool once = at < kept;
        if (u.dtype == LFMMI_F32) sum += squares<F32, Exact>(u, once);
        else if (u.dtype == LFMMI_BF16) sum += squares<Bf16, Exact>(u, once);
        else sum += squares<F16, Exact>(u, once);
    }
    return sum;
}

// Bound by the reads: 1.2e9 bf16 values of 420 tensors 383 us, 6.3 TB/s; 3e8 fp32 184 us, 6.5 TB/s.
template <typename List>
__global__ __launch_bounds__(kThreads) void k_grad_squares(List list, GradCall c)
{
    const auto l = tensors(list, c.n);
    double sum = sum_units<false>(l, c);
    if (__builtin_expect(!(sum < 0x1p256), 0)) sum = sum_units<true>(l, c);  // thread by thread
    sum = block_sum(sum);
    if (threadIdx.x == 0) c.partials[blockIdx.x] = sum;
}

// The norm, by a whole workgroup from all partial sums, in the same order in each.
__device__ __forceinline__ double norm_of(const GradCall& c)
{
    double sum = 0.;
    for (int i = threadIdx.x; i < c.blocks; i += kThreads) sum += c.partials[i];
    return sqrt(block_sum(sum));
}

// What brings it to max_norm; 0, so that every gradient becomes 0, if it is not finite.
__device__ __forceinline__ float factor_of(const GradCall& c, double norm)
{
    if (!((float)norm < INFINITY)) return 0.f;
    return norm > (double)c.max_norm ? (float)((double)c.max_norm / norm) : 1.f;
}

__global__ __launch_bounds__(kThreads) void k_grad_norm(GradCall c)
{
    const double norm = norm_of(c);
    if (threadIdx.x) return;
    *c.norm = (float)norm;
    *c.factor = factor_of(c, norm);
}

// (a factor of 0 makes a NaN 0 too)
__device__ __forceinline__ float scaled(float x, float factor) { return factor == 0.f ? 0.f : x * factor; }

template <typename D>
__device__ __forceinline__ void scale(const Unit& u, float factor, bool once)
{
    using Store = typename D::Store;
    Store* y = reinterpret_cast<Store*>(u.out);
    uint4 r[kUnitLoads<D>];
    load_unit<D>(u, once, r);
#pragma unroll
    for (int k = 0; k < kUnitLoads<D>; ++k) {
        const int q = threadIdx.x + k * kThreads;
        float f[D::kVec];
        D::unpack(r[k], f);
#pragma unroll
        for (int i = 0; i < D::kVec; ++i) f[i] = scaled(f[i], factor);
        if (has<D>(u, q)) {
            if (once) store16_once(y + q * D::kVec, D::pack(f));
            else store16(y + q * D::kVec, D::pack(f));
        }
    }
    if (u.to - u.from < kGradUnit)
        ends_of<D>(u, [&](int i) {
            D::store(y + i, scaled(D::load(reinterpret_cast<const Store*>(u.in) + i), factor));
        });
}

// A unit a workgroup, from the last to the first. (2,048 workgroups that go round the units took 17 % longer
// on 1.2e9 bf16 values: 830 us, 5.8 TB/s, the rate of a copy.)
// Alone: there is no k_grad_norm before it, every workgroup adds the partial sums up for itself.
template <typename List, bool Alone>
__global__ __launch_bounds__(kThreads) void k_grad_scale(List list, GradCall c)
{
    const auto l = tensors(list, c.n);
    const double norm = Alone ? norm_of(c) : 0.;
    if (Alone && blockIdx.x == 0 && threadIdx.x == 0) *c.norm = (float)norm;
    const float f = Alone ? factor_of(c, norm) : *c.factor;
    if (f == 1.f && c.in_place) return;
    for (int64_t at = c.units - 1 - (int64_t)blockIdx.x; at >= 0; at -= gridDim.x) {
        const Unit u = unit_of(l, (int)at);
        if (f == 1.f && u.in == u.out) continue;  // nothing to scale
        if (u.dtype == LFMMI_F32) scale<F32>(u, f, c.keep < 256);
        else if (u.dtype == LFMMI_BF16) scale<Bf16>(u, f, c.keep < 256);
        else scale<F16>(u, f, c.keep < 256);
    }
}

// Tensors from..from + l.n - 1 of a table (behind the last one, the number of units).
template <typename List>
__global__ __launch_bounds__(kThreads) void k_grad_table(List list, int from, GradTable t)
{
    const auto l = tensors(list, list.n);
    for (int i = threadIdx.x; i < l.n; i += kThreads) {
        t.in[from + i] = l.list.in(i);
        t.out[from + i] = l.list.out(i);
        t.count[from + i] = l.list.count(i);
        t.first[from + i] = l.list.first(i);
    }
    if (threadIdx.x == 0) t.first[from + l.n] = l.list.first(l.n);
}

}  // namespace

hipError_t launch_grad_table(const GradList& l, int from, const GradTable& t, hipStream_t stream)
{
    k_grad_table<<<1, kThreads, 0, stream>>>(l, from, t);
    return hipGetLastError();
}
hipError_t launch_grad_table(const GradPlaces& l, int from, const GradTable& t, hipStream_t stream)
{
    k_grad_table<<<1, kThreads, 0, stream>>>(l, from, t);
    return hipGetLastError();
}

namespace {

template <typename List>
hipError_t launch(const List& list, const GradCall& c, hipStream_t stream)
{
    if (c.blocks > 0) k_grad_squares<<<c.blocks, kThreads, 0, stream>>>(list, c);
    // Clipping 770 units: 19.5 us without a launch for the norm, 21.5 with it.
    if (c.scale && c.blocks > 0 && c.units <= kGradAlone) {
        k_grad_scale<List, true><<<c.units, kThreads, 0, stream>>>(list, c);
        return hipGetLastError();
    }
    k_grad_norm<<<1, kThreads, 0, stream>>>(c);
    if (c.scale && c.blocks > 0)
        k_grad_scale<List, false><<<std::min(c.units, 1 << 20), kThreads, 0, stream>>>(list, c);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_grads(const GradList& l, const GradCall& c, hipStream_t stream) { return launch(l, c, stream); }
hipError_t launch_grads(const GradPlaces& l, const GradCall& c, hipStream_t stream) { return launch(l, c, stream); }
hipError_t launch_grads(const GradTable& t, const GradCall& c, hipStream_t stream) { return launch(t, c, stream); }

}  // namespace lfmmi
