// Values of the types that the operators take, 16 bytes at a time.
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

namespace lfmmi {
namespace {

// 16 bytes a lane at any alignment of an element: rows of odd widths, views and pieces of buffers
// start anywhere (gfx950 takes such addresses; aligned ones lose nothing by it).
__device__ __forceinline__ uint4 load16(const void* p)
{
    uint4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
// ... of data that is not read again soon: it takes no place in the caches.
__device__ __forceinline__ uint4 load16_once(const void* p)
{
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
    typedef Words Anywhere __attribute__((aligned(2)));
    const Words v = __builtin_nontemporal_load(static_cast<const Anywhere*>(p));
    return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store16(void* p, uint4 v) { __builtin_memcpy(p, &v, 16); }
__device__ __forceinline__ void store16_once(void* p, uint4 v)
{
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
    typedef Words Anywhere __attribute__((aligned(2)));
    __builtin_nontemporal_store(Words{v.x, v.y, v.z, v.w}, static_cast<Anywhere*>(p));
}

typedef __bf16 Bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 F16x2 __attribute__((ext_vector_type(2)));

// Types of values: kVec of them in 16 bytes, kNone the bits of one word of -inf. Conversions to
// a 16-bit type round to nearest, ties to even.
struct F32 {
    using Store = float;
    static constexpr int kVec = 4;
    static constexpr uint32_t kNone = 0xff800000u;
    static __device__ __forceinline__ float load(const Store* p) { return *p; }
    static __device__ __forceinline__ void store(Store* p, float v) { *p = v; }
    static __device__ __forceinline__ void unpack(uint4 r, float* f)
    {
        f[0] = __uint_as_float(r.x);
        f[1] = __uint_as_float(r.y);
        f[2] = __uint_as_float(r.z);
        f[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ uint4 pack(const float* f)
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                          __float_as_uint(f[3]));
    }
};
struct Bf16 {
    using Store = uint16_t;
    static constexpr int kVec = 8;
    static constexpr uint32_t kNone = 0xff80ff80u;
    static __device__ __forceinline__ float load(const Store* p)
    {
        return __uint_as_float((uint32_t)*p << 16);
    }
    static __device__ __forceinline__ uint32_t pair(float a, float b)
    {
        return __builtin_bit_cast(uint32_t, Bf16x2{(__bf16)a, (__bf16)b});
    }
    static __device__ __forceinline__ void store(Store* p, float v)
    {
        *p = __builtin_bit_cast(uint16_t, (__bf16)v);
    }
    static __device__ __forceinline__ void unpack(uint4 r, float* f)
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint4 pack(const float* f)
    {
        return make_uint4(pair(f[0], f[1]), pair(f[2], f[3]), pair(f[4], f[5]), pair(f[6], f[7]));
    }
};
struct F16 {
    using Store = _Float16;
    static constexpr int kVec = 8;
    static constexpr uint32_t kNone = 0xfc00fc00u;
    static __device__ __forceinline__ float load(const Store* p) { return (float)*p; }
    static __device__ __forceinline__ uint32_t pair(float a, float b)
    {
        return __builtin_bit_cast(uint32_t, F16x2{(_Float16)a, (_Float16)b});
    }
    static __device__ __forceinline__ void store(Store* p, float v) { *p = (_Float16)v; }
    static __device__ __forceinline__ void unpack(uint4 r, float* f)
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)w[i]);
            f[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i] >> 16));
        }
    }
    static __device__ __forceinline__ uint4 pack(const float* f)
    {
        return make_uint4(pair(f[0], f[1]), pair(f[2], f[3]), pair(f[4], f[5]), pair(f[6], f[7]));
    }
};

}  // namespace
}  // namespace lfmmi
