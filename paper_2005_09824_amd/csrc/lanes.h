// Reductions over G lanes: 16 (a DPP row) or 64 (a wave); every lane has the result.
#pragma once
#include <hip/hip_runtime.h>

namespace lfmmi {
namespace {

template <int Ror>
__device__ __forceinline__ float rotated(float v)
{
    const int i = __float_as_int(v);
    return __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x120 + Ror, 0xf, 0xf, true));
}
__device__ __forceinline__ float lane_of(float v, int lane)
{
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

template <int G>
__device__ __forceinline__ float sum_over(float v)
{
    v += rotated<8>(v);
    v += rotated<4>(v);
    v += rotated<2>(v);
    v += rotated<1>(v);
    if (G == 64) v = (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
    return v;
}
template <int G>
__device__ __forceinline__ float max_over(float v)
{
    v = fmaxf(v, rotated<8>(v));
    v = fmaxf(v, rotated<4>(v));
    v = fmaxf(v, rotated<2>(v));
    v = fmaxf(v, rotated<1>(v));
    if (G == 64) v = fmaxf(fmaxf(lane_of(v, 0), lane_of(v, 16)), fmaxf(lane_of(v, 32), lane_of(v, 48)));
    return v;
}

}  // namespace
}  // namespace lfmmi
