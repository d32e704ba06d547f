// Rows of values, eight at a time, and the random bits that go with them.
#pragma once
#include <hip/hip_runtime.h>

#include "layers.h"
#include "vec16.h"

namespace lfmmi {
namespace {

// Eight values next to each other, of a row's `left` values from there on (what lies behind is 0).
template <typename T>
__device__ __forceinline__ void load8(const typename T::Store* p, int left, float* f)
{
    if (left >= 8) {
        T::unpack(load16(p), f);
        if (T::kVec == 4) T::unpack(load16(p + 4), f + 4);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < left ? T::load(p + i) : 0.f;
}
template <typename T>
__device__ __forceinline__ void store8(typename T::Store* p, int left, const float* f)
{
    if (left >= 8) {
        store16(p, T::pack(f));
        if (T::kVec == 4) store16(p + 4, T::pack(f + 4));
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) T::store(p + i, f[i]);
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
