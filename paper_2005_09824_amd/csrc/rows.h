// Rows of values, eight at a time, and the random bits that go with them.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "../../include/lfmmi.h"
#include "layers.h"
#include "vec16.h"

namespace lfmmi {
namespace {

// Eight values next to each other as they lie in memory, and unpacked.
template <typename T>
struct Raw {
    uint4 r[8 / T::kVec];
    __device__ __forceinline__ void unpack(float* f) const
    {
        T::unpack(r[0], f);
        if (T::kVec == 4) T::unpack(r[8 / T::kVec - 1], f + 4);
    }
};
template <typename T>
__device__ __forceinline__ Raw<T> no_values()
{
    Raw<T> v;
#pragma unroll
    for (int k = 0; k < 8 / T::kVec; ++k) v.r[k] = make_uint4(0, 0, 0, 0);
    return v;
}

// A row of fewer than eight values.
template <typename T>
__device__ __forceinline__ Raw<T> raw_short(const typename T::Store* p, int D)
{
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < D ? T::load(p + i) : 0.f;
    Raw<T> v;
#pragma unroll
    for (int k = 0; k < 8 / T::kVec; ++k) v.r[k] = T::pack(f + k * T::kVec);
    return v;
}

// Chunk c of a row of D values: columns 8 c and on. kWhole: eight divides D. kAny: otherwise, the last chunk is read as the
// row's last eight values, and moved to its place when it is unpacked. kShort: fewer than eight values. A branch around a load
// is waited for where it ends: a path of its own for the last chunk made 101 us of 83 (2,500 columns of bf16, 16,000 rows,
// forward), a look at D for short rows 152 of 146 (8,190 columns, 8,000 rows, backward).
enum Width { kAny, kWhole, kShort };
template <typename T, Width W>
__device__ __forceinline__ Raw<T> raw_at(const typename T::Store* row, int c, int D)
{
    if (W == kShort) return raw_short<T>(row, D);
    const typename T::Store* p = row + (W == kWhole ? c * 8 : min(c * 8, D - 8));
    Raw<T> v;
#pragma unroll
    for (int k = 0; k < 8 / T::kVec; ++k) v.r[k] = load16(p + k * T::kVec);
    return v;
}
template <int By>
__device__ __forceinline__ void move_down(float* f)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i + By < 8 ? f[i + By < 8 ? i + By : 0] : 0.f;
}
template <typename T, Width W>
__device__ __forceinline__ void unpack_at(const Raw<T>& v, int c, int D, float* f)
{
    v.unpack(f);
    if (W != kAny || c * 8 + 8 <= D) return;
    const int by = 8 - (D & 7);
    if (by & 4) move_down<4>(f);
    if (by & 2) move_down<2>(f);
    if (by & 1) move_down<1>(f);
}
template <typename T, Width W>
__device__ __forceinline__ void load_at(const typename T::Store* row, int c, int D, float* f)
{
    unpack_at<T, W>(raw_at<T, W>(row, c, D), c, D, f);
}
// (the values of a last chunk four, two and one at a time; once: past the caches, the same for all lanes. Eight values of 32 bits
// are two stores that each fill halves of lines, which the caches have to put together: 16,000 rows of 4,096 so 258 us, 194.)
template <typename T, Width W>
__device__ __forceinline__ void store_at(typename T::Store* row, int c, int D, const float* f, bool once = false)
{
    typename T::Store* p = row + c * 8;
    const int left = D - c * 8;
    uint4 r[8 / T::kVec];
#pragma unroll
    for (int k = 0; k < 8 / T::kVec; ++k) r[k] = T::pack(f + k * T::kVec);
    if (W == kWhole || left >= 8) {
#pragma unroll
        for (int k = 0; k < 8 / T::kVec; ++k) {
            if (once && T::kVec == 8) {
                asm volatile("");  // (two stores that differ by a hint alone are made one without it)
                store16_once(p + k * T::kVec, r[k]);
                asm volatile("");
            } else {
                store16(p + k * T::kVec, r[k]);
            }
        }
        return;
    }
    if constexpr (T::kVec == 4) {
        const uint4 rest = left & 4 ? r[1] : r[0];
        if (left & 4) store16(p, r[0]);
        if (left & 2) __builtin_memcpy(p + (left & 4), &rest, 8);
        const uint32_t one = left & 2 ? rest.z : rest.x;
        if (left & 1) __builtin_memcpy(p + left - 1, &one, 4);
    } else {
        if (left & 4) __builtin_memcpy(p, &r[0], 8);
        const uint32_t two = left & 4 ? r[0].z : r[0].x, next = left & 4 ? r[0].w : r[0].y;
        if (left & 2) __builtin_memcpy(p + (left & 4), &two, 4);
        const uint16_t one = (uint16_t)(left & 2 ? next : two);
        if (left & 1) __builtin_memcpy(p + left - 1, &one, 2);
    }
}

// Calls f with the kind of a width, as a type; kShort where rows of fewer than eight values come here at all.
template <bool Short, typename F>
void by_width(int D, F&& f)
{
    if (D % 8 == 0) f(std::integral_constant<Width, kWhole>{});
    else if (Short && D < 8) f(std::integral_constant<Width, Short ? kShort : kAny>{});
    else f(std::integral_constant<Width, kAny>{});
}
template <typename F>
void by_type(int dtype, F&& f)
{
    if (dtype == LFMMI_F32) f(F32{});
    else if (dtype == LFMMI_BF16) f(Bf16{});
    else f(F16{});
}

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, SC 2011):
// ten rounds of two products of 32 bits on a counter of 128 bits.
struct Words {
    uint32_t w[4];
};
__device__ __forceinline__ Words philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)b;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// What is kept of the eight values of columns 8 * chunk and on of a row, times `factor`; 16 bits a
// value. What is dropped is 0, whatever it was.
struct Dropping {
    uint32_t k0, k1, c2, c3;
    uint32_t threshold;
    float factor;
    __device__ __forceinline__ explicit Dropping(const Draw& d)
    {
        const uint64_t draw = d.threshold > 0 && d.step ? d.offset + (uint64_t)*d.step : d.offset;
        k0 = (uint32_t)d.seed;
        k1 = (uint32_t)(d.seed >> 32);
        c2 = (uint32_t)draw;
        c3 = (uint32_t)(draw >> 32);
        threshold = (uint32_t)d.threshold;
        factor = d.factor;
    }
    __device__ __forceinline__ void apply(uint32_t row, uint32_t chunk, float* f) const
    {
        const Words r = philox(chunk, row, c2, c3, k0, k1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t bits = i & 1 ? r.w[i >> 1] >> 16 : r.w[i >> 1] & 0xffffu;
            f[i] = bits >= threshold ? f[i] * factor : 0.f;
        }
    }
};

}  // namespace
}  // namespace lfmmi
