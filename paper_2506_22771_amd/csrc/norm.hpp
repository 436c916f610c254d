// Host-side launchers of the layer norm, the 8-bit checkpoints and the weight gradient read from them.
#pragma once

#include "ff_internal.hpp"

namespace ffi {

struct NormForwardLaunch {
    const void* x;
    int64_t ldx;
    const void* weight;   // may be null
    const void* bias;     // may be null
    void* y;
    int64_t ldy;
    float* mean;          // may be null
    float* rstd;          // may be null
    int64_t rows, cols;
    int32_t dtype, param_dtype;
    float eps;
    int8_t* q;            // checkpoint of the normalised rows, or null
    uint8_t* e;
    int32_t round_mode;
    uint64_t seed, tag;
};
hipError_t launch_norm_forward(const NormForwardLaunch& a, hipStream_t s);

struct NormBackwardLaunch {
    const void* dy;
    int64_t lddy;
    const void* x;        // null: the checkpoint is read
    int64_t ldx;
    const float* mean;
    const int8_t* q;
    const uint8_t* e;
    const float* rstd;
    const void* weight;   // may be null
    void* dx;             // may be null
    int64_t lddx;
    float* dweight;       // may be null
    float* dbias;         // may be null
    int64_t rows, cols;
    int32_t dtype, param_dtype, accumulate;
    void* ws;
};
size_t norm_backward_workspace(int64_t rows, int64_t cols);
hipError_t launch_norm_backward(const NormBackwardLaunch& a, hipStream_t s);

hipError_t launch_ckpt_store(const void* x, int32_t dtype, int64_t ldx, int64_t rows, int64_t cols, int32_t round_mode, uint64_t seed,
                             uint64_t tag, int8_t* q, uint8_t* e, hipStream_t s);
hipError_t launch_ckpt_load(const int8_t* q, const uint8_t* e, int64_t rows, int64_t cols, void* x, int32_t dtype, int64_t ldx,
                            hipStream_t s);
hipError_t launch_ckpt_act_backward(const int8_t* q, const uint8_t* e, int64_t rows, int64_t cols, int32_t act, const float* coeff,
                                    const void* dy, int64_t lddy, void* dx, int64_t lddx, int32_t dtype, hipStream_t s);

struct CkptWgradLaunch {
    const void* dy;
    int64_t lddy;
    int32_t dtype;
    const int8_t* q;
    const uint8_t* e;
    int64_t rows, n, k;
    const void* gamma;    // may be null
    const void* beta;     // may be null
    int32_t param_dtype;
    float* dw;
    float* db;            // may be null
    int32_t accumulate;
    void* ws;
};
size_t ckpt_wgrad_workspace(int64_t rows, int64_t n, int64_t k);
hipError_t launch_ckpt_wgrad(const CkptWgradLaunch& a, hipStream_t s);

}  // namespace ffi
