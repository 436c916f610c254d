// C-ABI entry points of the gated layer, the group norm and dropout: argument validation on the host, then the launches on the caller's stream.
#include "api_checks.hpp"
#include "blocks.hpp"

using namespace ffi;

static bool act_ok(int32_t act) { return act >= FF_ACT_IDENTITY && act <= FF_ACT_SILU; }

extern "C" {

static ff_status gated_size_status(int64_t rows, int64_t n, int64_t k)
{
    if (rows < 0 || n < 0 || k < 0) return FF_ERR_INVALID_ARG;
    if (n == 0 || k == 0) return FF_ERR_SHAPE;
    if (n > 65535 / 2 || rows > 8388480) return FF_ERR_UNSUPPORTED;   // features and rows of quantised matrices, as everywhere in this interface
    if (k > INT32_MAX / (127 * 127)) return FF_ERR_OVERFLOW_BOUND;
    return size_status(rows, n);
}

size_t ff_gated_workspace_bytes(int64_t rows, int64_t n, int64_t k)
{
    return gated_size_status(rows, n, k) == FF_OK ? gated_workspace(rows, n, k) : 0;
}

ff_status ff_gated_forward(int64_t rows, int64_t n, int64_t k, const int8_t* a_q, const int8_t* w_q, const float* s_a, const float* s_w, int32_t act,
                           void* y, int32_t dtype, int64_t ldy, float* goodness, int8_t* qg, uint8_t* eg, int8_t* qu, uint8_t* eu, void* ws,
                           size_t ws_bytes, void* stream)
{
    REFUSE(gated_size_status(rows, n, k));
    if (!type_ok(dtype) || !act_ok(act) || !w_q || !s_a || !s_w || !ws) return FF_ERR_INVALID_ARG;
    if (ws_bytes < gated_workspace(rows, n, k)) return FF_ERR_WORKSPACE;
    if (!aligned16(ws) || !aligned16(a_q) || !aligned16(w_q) || !aligned4(s_a) || !aligned4(s_w) || !aligned4(goodness)) return FF_ERR_ALIGN;
    if (rows == 0) return FF_OK;
    if (!a_q) return FF_ERR_INVALID_ARG;
    REFUSE(matrix_status(y, dtype, ldy, n));
    if (qg || eg || qu || eu) {
        REFUSE(ckpt_status(qg, eg));
        REFUSE(ckpt_status(qu, eu));
    }
    hipStream_t s = (hipStream_t)stream;
    HIPCHK_T(FF_K_GATED, launch_gated_forward({a_q, w_q, s_a, s_w, rows, n, k, act, dtype, y, ldy, goodness, qg, eg, qu, eu, ws}, s));
    return FF_OK;
}

ff_status ff_gated_backward(const int8_t* qg, const uint8_t* eg, const int8_t* qu, const uint8_t* eu, int64_t rows, int64_t n, int32_t act,
                            const float* coeff, const void* dy, int64_t lddy, void* dg, int64_t lddg, void* du, int64_t lddu, int32_t dtype,
                            void* stream)
{
    REFUSE(size_status(rows, n));
    if (!type_ok(dtype) || !act_ok(act)) return FF_ERR_INVALID_ARG;
    if (rows == 0) return FF_OK;
    if (!coeff && !dy) return FF_ERR_INVALID_ARG;
    if (!aligned4(coeff)) return FF_ERR_ALIGN;
    REFUSE(ckpt_status(qg, eg));
    REFUSE(ckpt_status(qu, eu));
    if (dy) REFUSE(matrix_status(dy, dtype, lddy, n));
    REFUSE(matrix_status(dg, dtype, lddg, n));
    REFUSE(matrix_status(du, dtype, lddu, n));
    hipStream_t s = (hipStream_t)stream;
    HIPCHK_T(FF_K_GATED, launch_gated_backward({qg, eg, qu, eu, rows, n, act, dtype, coeff, dy, dg, du, lddy, lddg, lddu}, s));
    return FF_OK;
}

static ff_status group_size_status(int64_t samples, int64_t pixels, int64_t channels, int64_t groups)
{
    if (samples < 0 || pixels < 0 || channels < 0 || groups < 0) return FF_ERR_INVALID_ARG;
    if (pixels == 0 || channels == 0 || groups == 0 || channels % groups != 0) return FF_ERR_SHAPE;
    if (channels > 65535 || samples > MOST_ROWS || pixels > MOST_ROWS || samples * pixels > MOST_ROWS) return FF_ERR_UNSUPPORTED;
    return size_status(samples * pixels, channels);
}

size_t ff_group_norm_workspace_bytes(int64_t samples, int64_t pixels, int64_t channels, int64_t groups)
{
    return group_size_status(samples, pixels, channels, groups) == FF_OK ? group_norm_workspace(samples, pixels, channels, groups) : 0;
}

ff_status ff_group_norm_forward(int64_t samples, int64_t pixels, int64_t channels, int64_t groups, int32_t dtype, int32_t param_dtype, const void* x,
                                int64_t ldx, const void* weight, const void* bias, float eps, int32_t act, void* y, int64_t ldy, float* mean,
                                float* rstd, float* goodness, int8_t* q, uint8_t* e, int32_t round_mode, uint64_t seed, uint64_t stream_tag,
                                void* ws, size_t ws_bytes, void* stream)
{
    REFUSE(group_size_status(samples, pixels, channels, groups));
    if (!type_ok(dtype) || (param_dtype != FF_F32 && param_dtype != dtype) || !act_ok(act) || !(eps >= 0.0f) || !round_ok(round_mode) || !ws)
        return FF_ERR_INVALID_ARG;
    if (ws_bytes < group_norm_workspace(samples, pixels, channels, groups)) return FF_ERR_WORKSPACE;
    if (!aligned16(ws) || !aligned_to(weight, param_dtype) || !aligned_to(bias, param_dtype) || !aligned4(mean) || !aligned4(rstd) || !aligned4(goodness))
        return FF_ERR_ALIGN;
    if (samples == 0) return FF_OK;
    REFUSE(matrix_status(x, dtype, ldx, channels));
    REFUSE(matrix_status(y, dtype, ldy, channels));
    if (q || e) REFUSE(ckpt_status(q, e));
    hipStream_t s = (hipStream_t)stream;
    HIPCHK_T(FF_K_GROUP_NORM, launch_group_norm_forward({samples, pixels, channels, groups, dtype, param_dtype, act, x, ldx, weight, bias, eps, y, ldy,
                                                         mean, rstd, goodness, q, e, round_mode, seed, stream_tag, ws}, s));
    return FF_OK;
}

ff_status ff_group_norm_backward(int64_t samples, int64_t pixels, int64_t channels, int64_t groups, int32_t dtype, int32_t param_dtype, const void* dy,
                                 int64_t lddy, const float* coeff, const void* x, int64_t ldx, const float* mean, const int8_t* q, const uint8_t* e,
                                 const float* rstd, const void* weight, const void* bias, int32_t act, void* dx, int64_t lddx, float* dweight,
                                 float* dbias, int32_t accumulate, void* ws, size_t ws_bytes, void* stream)
{
    REFUSE(group_size_status(samples, pixels, channels, groups));
    if (!type_ok(dtype) || (param_dtype != FF_F32 && param_dtype != dtype) || !act_ok(act) || (accumulate != 0 && accumulate != 1) || !ws ||
        (!dx && !dweight && !dbias))
        return FF_ERR_INVALID_ARG;
    if (ws_bytes < group_norm_workspace(samples, pixels, channels, groups)) return FF_ERR_WORKSPACE;
    if (!aligned16(ws) || !aligned_to(weight, param_dtype) || !aligned_to(bias, param_dtype) || !aligned4(coeff) || !aligned4(mean) || !aligned4(rstd) ||
        !aligned4(dweight) || !aligned4(dbias))
        return FF_ERR_ALIGN;
    if (samples > 0) {
        if (!coeff && !dy) return FF_ERR_INVALID_ARG;
        if (dy) REFUSE(matrix_status(dy, dtype, lddy, channels));
        if (x) REFUSE(matrix_status(x, dtype, ldx, channels));
        else REFUSE(ckpt_status(q, e));
        if (dx) REFUSE(matrix_status(dx, dtype, lddx, channels));
        if (!rstd || (x && !mean)) return FF_ERR_INVALID_ARG;
    }
    hipStream_t s = (hipStream_t)stream;
    HIPCHK_T(FF_K_GROUP_NORM, launch_group_norm_backward({samples, pixels, channels, groups, dtype, param_dtype, act, coeff, dy, lddy, x, ldx, mean, q, e, rstd,
                                                          weight, bias, dx, lddx, dweight, dbias, accumulate, ws}, s));
    return FF_OK;
}

ff_status ff_dropout(int64_t rows, int64_t cols, int32_t dtype, const void* x, int64_t ldx, const void* r, int64_t ldr, float p, uint64_t seed,
                     uint64_t stream_tag, const uint64_t* step_dev, void* y, int64_t ldy, void* stream)
{
    REFUSE(size_status(rows, cols));
    if (!type_ok(dtype) || !(p >= 0.0f && p <= 1.0f)) return FF_ERR_INVALID_ARG;
    if ((uintptr_t)step_dev & 7) return FF_ERR_ALIGN;
    if (rows == 0) return FF_OK;
    REFUSE(matrix_status(x, dtype, ldx, cols));
    if (r) REFUSE(matrix_status(r, dtype, ldr, cols));
    REFUSE(matrix_status(y, dtype, ldy, cols));
    hipStream_t s = (hipStream_t)stream;
    HIPCHK_T(FF_K_DROPOUT, launch_dropout({x, r, y, ldx, ldr, ldy, rows, cols, dtype, p, seed, stream_tag, step_dev}, s));
    return FF_OK;
}

}  // extern "C"
