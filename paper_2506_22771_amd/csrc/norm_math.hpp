// Arithmetic shared by the layer norm (norm.hip) and the group norm (group_norm.hip).
#pragma once

#include "ckpt.hpp"

namespace ffi {

// 1 / sqrt(v) to one unit in the last place; the instruction takes no numbers below 2^-126.
__device__ __forceinline__ float inverse_root(float v)
{
    const bool low = v < 0x1p-96f;
    const float r = __builtin_amdgcn_rsqf(low ? v * 0x1p96f : v);
    return low ? r * 0x1p48f : r;
}

// What is left of a row's mean, by the mean of the deviations from it and that of their squares; and the variance.  (Not below zero by a rounding; NaN stays.)
__device__ __forceinline__ float mean_rest(float mean, float deviation, float square) { return mean * mean > square ? deviation : 0.0f; }
__device__ __forceinline__ float variance(float square, float rest)
{
    const float v = __builtin_fmaf(-rest, rest, square);
    return v < 0 ? 0.0f : v;
}

// Eight parameters of a chunk (n of them exist), in the element's type or in fp32; `none` where there are none.
template <typename T> __device__ __forceinline__ void load_param(const void* p, bool f32, int64_t at, int n, float none, float v[8])
{
    if (p == nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = none;
    } else if (sizeof(T) == 4 || f32) {
        load8((const float*)p + at, n, v);
    } else {
        load8((const T*)p + at, n, v);
    }
}

}  // namespace ffi
