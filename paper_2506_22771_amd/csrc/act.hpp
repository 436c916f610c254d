// Activation functions with their derivatives, for values of type T (what they are rounded to decides how close they are).
#pragma once

#include "ckpt.hpp"

namespace ffi {

// f(u) and f'(u).  GELU's exponential is the density's as well as a factor of Phi(-|u|).
// 16-bit values, where f' is the output (not ANY): Phi(-|u|) = 1/2 t (a1 + t (a2 + ...)) exp(-u^2/2), t = 1 / (1 + p |u| / sqrt 2): Abramowitz and Stegun 7.1.26, off by at
// most 0.75e-7, and f' by no more than that.  With more arithmetic than this the large case is bound by it and not by memory: 16384 x 4096 bf16 values 96 us with
// the library's erf and exp, 62 to 65 this way.
// 16-bit values, where f is an output or the gradient goes into fp32 sums (ANY): far below zero f = u Phi(u) is as small as Phi, of which that sum is off by 6e-4 at u = -4.2 and
// 4e-3 at -6, more than half a step of fp16 and of bf16.  One term more, fitted to errors relative to Phi as well: off by at most 1.1e-8, and by 2.8e-5 of Phi down to -6, 6e-4 down
// to -9.  (rms of f' 6.1e-8 of its size, by the shorter sum 9.9e-8.  16384 x 4096 bf16, the gated layer's gradient, 97 us and 96 by the shorter sum; 512 x 32x32 x 128 bf16 group norm
// backward from x 152 and 147, from codes 131 and 130, forward 69 either way.)
// fp32 values: the shorter sum is off by more than the rounding of an fp32 product (rms of f' 9.7e-8 of its size), so Phi = 1/2 + u P(u^2) up to |u| = 1.25, off by at most 2.1e-9, and
// Phi(-|u|) = t Q(t) exp(-u^2/2), t = 1 / (1 + 0.3 |u|), beyond, off by at most 4.3e-9; P and Q are least-squares fits, reweighted towards the smallest largest
// error (rms of f' 4.0e-8; with the device library's erf 4.1e-8, and 16384 x 4096 values with goodness 114 us, 120 that way, 109 by the shorter sum and with ReLU).
// SiLU of fp32 values (OUT): the exponential's argument x = -u log2(e) is a rounded product, whose error grows with it (f off by 1.7e-6 of itself at u = -60).  What the rounding
// left, c = -u - x ln 2, goes into it as exp(-u) = 2^x (1 + c).  Where f goes into an output by its derivative alone it is left out (the group norm's gradient, 512 x 4x4 x 512:
// 18.1 us, with it 18.7).
// ANY: of any fp32 argument; else of what a checkpoint holds, for the gradient.  OUT: f is an output, or a factor of one.
template <typename T, int ACT, bool ANY = false, bool OUT = ANY> __device__ __forceinline__ void act_of(float u, float& f, float& d)
{
    if constexpr (ACT == FF_ACT_RELU) {
        f = u <= 0 ? 0.0f : u;   // (NaN stays)
        d = u > 0 ? 1.0f : (u == u ? 0.0f : u);
    } else if constexpr (ACT == FF_ACT_GELU) {
        const float e = __builtin_amdgcn_exp2f(u * u * -0.72134752044448170f);              // exp(-u^2 / 2)
        float phi;
        if constexpr (sizeof(T) == 4) {
            const float s = u * u, t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(u), 0.3f, 1.0f));
            float p = __builtin_fmaf(s, -6.64486e-6f, 1.1032746e-4f);
            p = __builtin_fmaf(s, p, -1.1827096e-3f);
            p = __builtin_fmaf(s, p, 9.9715004e-3f);
            p = __builtin_fmaf(s, p, -0.06648999f);
            p = __builtin_fmaf(s, p, 0.39894226f);
            float q = __builtin_fmaf(t, -0.033505592f, 0.30637836f);
            q = __builtin_fmaf(t, q, -0.06527595f);
            q = __builtin_fmaf(t, q, 0.18152371f);
            q = __builtin_fmaf(t, q, 0.11132239f);
            const float low = t * q * e;
            phi = __builtin_fabsf(u) < 1.25f ? __builtin_fmaf(u, p, 0.5f) : u > 0 ? 1.0f - low : low;
        } else if constexpr (ANY) {
            const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(u), 0.281f, 1.0f));
            float q = __builtin_fmaf(t, -0.103819676f, 0.377323121f);
            q = __builtin_fmaf(t, q, -0.218507633f);
            q = __builtin_fmaf(t, q, 0.256346375f);
            q = __builtin_fmaf(t, q, 0.0723568052f);
            q = __builtin_fmaf(t, q, 0.116301f);
            const float low = t * q * e;
            phi = u > 0 ? 1.0f - low : low;
        } else {
            const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(u), 0.23164189110f, 1.0f));   // p / sqrt 2
            float q = __builtin_fmaf(t, 0.5307027145f, -0.7265760135f);                     // half of the polynomial
            q = __builtin_fmaf(t, q, 0.7107068705f);
            q = __builtin_fmaf(t, q, -0.142248368f);
            q = __builtin_fmaf(t, q, 0.127414796f);
            // Phi(u): 1 - low above zero, else low; a code that is not zero stands for 2^-106 at least
            phi = __builtin_fabsf(__builtin_amdgcn_fmed3f(u * 0x1p127f, 0.0f, 1.0f) - t * q * e);
        }
        f = u * phi;
        d = __builtin_fmaf(u * e, 0.39894228040143268f, phi);
    } else if constexpr (ACT == FF_ACT_SILU) {
        float e;
        if constexpr (OUT && sizeof(T) == 4) {
            const float v = __builtin_amdgcn_fmed3f(u, -88.72283f, 88.72283f), x = v * -1.4426950408889634f;   // (e is finite; beyond, sigma is 0 or 1)
            e = __builtin_amdgcn_exp2f(x);
            e = __builtin_fmaf(e, __builtin_fmaf(x, -0.693147182f, -v), e);
        } else {
            e = __builtin_amdgcn_exp2f(u * -1.4426950408889634f);
        }
        const float sig = __builtin_amdgcn_rcpf(1.0f + e);
        f = u * sig;
        d = __builtin_fmaf(f, 1.0f - sig, sig);
    } else {
        f = u;
        d = 1.0f;
    }
}

}  // namespace ffi
