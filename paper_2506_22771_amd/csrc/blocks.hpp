// Host-side launchers of the gated layer, the group norm and dropout.
#pragma once

#include "ff_internal.hpp"

namespace ffi {

struct DropoutLaunch {
    const void* x;
    const void* r;      // may be null
    void* y;
    int64_t ldx, ldr, ldy, rows, cols;
    int32_t dtype;
    float p;
    uint64_t seed, tag;
    const uint64_t* step_dev;   // may be null
};
hipError_t launch_dropout(const DropoutLaunch& a, hipStream_t s);

struct GatedForwardLaunch {
    const int8_t* a_q;
    const int8_t* w_q;
    const float* s_a;
    const float* s_w;
    int64_t rows, n, k;
    int32_t act, dtype;
    void* y;
    int64_t ldy;
    float* goodness;    // may be null
    int8_t* qg;         // all four or none
    uint8_t* eg;
    int8_t* qu;
    uint8_t* eu;
    void* ws;
};
size_t gated_workspace(int64_t rows, int64_t n, int64_t k);
hipError_t launch_gated_forward(const GatedForwardLaunch& a, hipStream_t s);

struct GatedBackwardLaunch {
    const int8_t* qg;
    const uint8_t* eg;
    const int8_t* qu;
    const uint8_t* eu;
    int64_t rows, n;
    int32_t act, dtype;
    const float* coeff;   // may be null
    const void* dy;       // may be null
    void* dg;
    void* du;
    int64_t lddy, lddg, lddu;
};
hipError_t launch_gated_backward(const GatedBackwardLaunch& a, hipStream_t s);

struct GroupNormForwardLaunch {
    int64_t samples, pixels, channels, groups;
    int32_t dtype, param_dtype, act;
    const void* x;
    int64_t ldx;
    const void* weight;   // may be null
    const void* bias;     // may be null
    float eps;
    void* y;
    int64_t ldy;
    float* mean;          // may be null
    float* rstd;          // may be null
    float* goodness;      // may be null
    int8_t* q;            // checkpoint of the normalised maps, or null
    uint8_t* e;
    int32_t round_mode;
    uint64_t seed, tag;
    void* ws;
};
struct GroupNormBackwardLaunch {
    int64_t samples, pixels, channels, groups;
    int32_t dtype, param_dtype, act;
    const float* coeff;   // may be null
    const void* dy;       // may be null
    int64_t lddy;
    const void* x;        // null: the checkpoint is read
    int64_t ldx;
    const float* mean;
    const int8_t* q;
    const uint8_t* e;
    const float* rstd;
    const void* weight;   // may be null
    const void* bias;     // may be null
    void* dx;             // may be null
    int64_t lddx;
    float* dweight;       // may be null
    float* dbias;         // may be null
    int32_t accumulate;
    void* ws;
};
size_t group_norm_workspace(int64_t samples, int64_t pixels, int64_t channels, int64_t groups);
hipError_t launch_group_norm_forward(const GroupNormForwardLaunch& a, hipStream_t s);
hipError_t launch_group_norm_backward(const GroupNormBackwardLaunch& a, hipStream_t s);

}  // namespace ffi
