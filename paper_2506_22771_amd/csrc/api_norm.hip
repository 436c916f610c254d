// C-ABI entry points of the layer norm and the 8-bit checkpoints: argument validation on the host, then the launches on the
// caller's stream.
#include "norm.hpp"

namespace ffi {

constexpr int64_t MOST_COLS = int64_t(1) << 24, MOST_ROWS = (int64_t(1) << 31) - 1, MOST_LD = int64_t(1) << 31;

static ff_status size_status(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0) return FF_ERR_INVALID_ARG;
    if (cols == 0) return FF_ERR_SHAPE;
    if (cols > MOST_COLS || rows > MOST_ROWS) return FF_ERR_UNSUPPORTED;
    // chunks of eight columns, whole blocks of them; a launch has fewer than 2^32 lanes, at most two for a chunk
    if (rows * ((pitch8(cols) + 31) / 32 * 4) >= int64_t(1) << 31) return FF_ERR_UNSUPPORTED;
    return FF_OK;
}
static bool type_ok(int32_t t) { return t == FF_F32 || t == FF_BF16 || t == FF_F16; }
static bool round_ok(int32_t r) { return r == FF_ROUND_NEAREST_EVEN || r == FF_ROUND_STOCHASTIC; }
static bool aligned_to(const void* p, int32_t type) { return ((uintptr_t)p & (type == FF_F32 ? 3 : 1)) == 0; }
// a matrix that has to be there (rows > 0)
static ff_status matrix_status(const void* p, int32_t type, int64_t ld, int64_t cols)
{
    if (!p) return FF_ERR_INVALID_ARG;
    if (ld < cols) return FF_ERR_SHAPE;
    if (ld > MOST_LD) return FF_ERR_UNSUPPORTED;
    return aligned_to(p, type) ? FF_OK : FF_ERR_ALIGN;
}
static ff_status ckpt_status(const void* q, const void* e)
{
    if (!q || !e) return FF_ERR_INVALID_ARG;
    return aligned16(q) && aligned16(e) ? FF_OK : FF_ERR_ALIGN;
}
#define REFUSE(e) do { const ff_status _st = (e); if (_st != FF_OK) return _st; } while (0)

}  // namespace ffi

using namespace ffi;

extern "C" {

int64_t ff_ckpt_blocks(int64_t cols) { return cols <= 0 ? 0 : (cols + FF_CKPT_BLOCK - 1) / FF_CKPT_BLOCK; }

ff_status ff_layer_norm_forward(int64_t rows, int64_t cols, int32_t dtype, int32_t param_dtype, const void* x, int64_t ldx,
                                const void* weight, const void* bias, float eps, void* y, int64_t ldy, float* mean,
                                float* rstd, int8_t* q, uint8_t* e, int32_t round_mode, uint64_t seed,
                                uint64_t stream_tag, void* stream)
{
    REFUSE(size_status(rows, cols));
    if (!type_ok(dtype) || (param_dtype != FF_F32 && param_dtype != dtype) || !(eps >= 0.0f) || !round_ok(round_mode))
        return FF_ERR_INVALID_ARG;
    if (!aligned_to(weight, param_dtype) || !aligned_to(bias, param_dtype) || !aligned4(mean) || !aligned4(rstd)) return FF_ERR_ALIGN;
    if (rows == 0) return FF_OK;
    REFUSE(matrix_status(x, dtype, ldx, cols));
    REFUSE(matrix_status(y, dtype, ldy, cols));
    if (q || e) REFUSE(ckpt_status(q, e));
    hipStream_t s = (hipStream_t)stream;
    HIPCHK_T(FF_K_NORM, launch_norm_forward({x, ldx, weight, bias, y, ldy, mean, rstd, rows, cols, dtype, param_dtype, eps, q, e,
                                             round_mode, seed, stream_tag}, s));
    return FF_OK;
}

size_t ff_layer_norm_workspace_bytes(int64_t rows, int64_t cols)
{
    return size_status(rows, cols) == FF_OK ? norm_backward_workspace(rows, cols) : 0;
}

ff_status ff_layer_norm_backward(int64_t rows, int64_t cols, int32_t dtype, int32_t param_dtype, const void* dy,
                                 int64_t lddy, const void* x, int64_t ldx, const float* mean, const int8_t* q,
                                 const uint8_t* e, const float* rstd, const void* weight, void* dx, int64_t lddx,
                                 float* dweight, float* dbias, int32_t accumulate, void* ws, size_t ws_bytes,
                                 void* stream)
{
    REFUSE(size_status(rows, cols));
    if (!type_ok(dtype) || (param_dtype != FF_F32 && param_dtype != dtype) || (accumulate != 0 && accumulate != 1) || !ws ||
        (!dx && !dweight && !dbias))
        return FF_ERR_INVALID_ARG;
    if (ws_bytes < norm_backward_workspace(rows, cols)) return FF_ERR_WORKSPACE;
    if (!aligned16(ws) || !aligned_to(weight, param_dtype) || !aligned4(mean) || !aligned4(rstd) || !aligned4(dweight) || !aligned4(dbias))
        return FF_ERR_ALIGN;
    if (rows > 0) {
        REFUSE(matrix_status(dy, dtype, lddy, cols));
        if (x) REFUSE(matrix_status(x, dtype, ldx, cols));
        else REFUSE(ckpt_status(q, e));
        if (dx) REFUSE(matrix_status(dx, dtype, lddx, cols));
        if (!rstd || (x && !mean)) return FF_ERR_INVALID_ARG;
    }
    hipStream_t s = (hipStream_t)stream;
    HIPCHK_T(FF_K_NORM, launch_norm_backward({dy, lddy, x, ldx, mean, q, e, rstd, weight, dx, lddx, dweight, dbias, rows, cols, dtype,
                                              param_dtype, accumulate, ws}, s));
    return FF_OK;
}

ff_status ff_ckpt_store(const void* x, int32_t dtype, int64_t ldx, int64_t rows, int64_t cols, int32_t round_mode,
                        uint64_t seed, uint64_t stream_tag, int8_t* q, uint8_t* e, void* stream)
{
    REFUSE(size_status(rows, cols));
    if (!type_ok(dtype) || !round_ok(round_mode)) return FF_ERR_INVALID_ARG;
    if (rows == 0) return FF_OK;
    REFUSE(matrix_status(x, dtype, ldx, cols));
    REFUSE(ckpt_status(q, e));
    hipStream_t s = (hipStream_t)stream;
    HIPCHK_T(FF_K_CKPT, launch_ckpt_store(x, dtype, ldx, rows, cols, round_mode, seed, stream_tag, q, e, s));
    return FF_OK;
}

ff_status ff_ckpt_load(const int8_t* q, const uint8_t* e, int64_t rows, int64_t cols, void* x, int32_t dtype, int64_t ldx,
                       void* stream)
{
    REFUSE(size_status(rows, cols));
    if (!type_ok(dtype)) return FF_ERR_INVALID_ARG;
    if (rows == 0) return FF_OK;
    REFUSE(ckpt_status(q, e));
    REFUSE(matrix_status(x, dtype, ldx, cols));
    hipStream_t s = (hipStream_t)stream;
    HIPCHK_T(FF_K_CKPT, launch_ckpt_load(q, e, rows, cols, x, dtype, ldx, s));
    return FF_OK;
}

ff_status ff_ckpt_act_backward(const int8_t* q, const uint8_t* e, int64_t rows, int64_t cols, int32_t act,
                               const float* coeff, const void* dy, int64_t lddy, void* dx, int64_t lddx, int32_t dtype,
                               void* stream)
{
    REFUSE(size_status(rows, cols));
    if (!type_ok(dtype) || act < FF_ACT_IDENTITY || act > FF_ACT_SILU) return FF_ERR_INVALID_ARG;
    if (rows == 0) return FF_OK;
    if (!coeff && !dy) return FF_ERR_INVALID_ARG;
    if (!aligned4(coeff)) return FF_ERR_ALIGN;
    REFUSE(ckpt_status(q, e));
    if (dy) REFUSE(matrix_status(dy, dtype, lddy, cols));
    REFUSE(matrix_status(dx, dtype, lddx, cols));
    hipStream_t s = (hipStream_t)stream;
    HIPCHK_T(FF_K_CKPT, launch_ckpt_act_backward(q, e, rows, cols, act, coeff, dy, lddy, dx, lddx, dtype, s));
    return FF_OK;
}

static ff_status wgrad_size_status(int64_t rows, int64_t n, int64_t k)
{
    REFUSE(size_status(rows, k));
    REFUSE(size_status(rows, n));
    return n > 65535 ? FF_ERR_UNSUPPORTED : FF_OK;   // as everywhere in this interface
}

size_t ff_ckpt_weight_grad_workspace_bytes(int64_t rows, int64_t n, int64_t k)
{
    return wgrad_size_status(rows, n, k) == FF_OK ? ckpt_wgrad_workspace(rows, n, k) : 0;
}

ff_status ff_ckpt_weight_grad(const void* dy, int32_t dtype, int64_t lddy, const int8_t* q, const uint8_t* e, int64_t rows,
                              int64_t n, int64_t k, const void* gamma, const void* beta, int32_t param_dtype, float* dw,
                              float* db, int32_t accumulate, void* ws, size_t ws_bytes, void* stream)
{
    REFUSE(wgrad_size_status(rows, n, k));
    if (!type_ok(dtype) || (param_dtype != FF_F32 && param_dtype != dtype) || (accumulate != 0 && accumulate != 1) || !dw || !ws)
        return FF_ERR_INVALID_ARG;
    if (ws_bytes < ckpt_wgrad_workspace(rows, n, k)) return FF_ERR_WORKSPACE;
    if (!aligned16(ws) || !aligned_to(gamma, param_dtype) || !aligned_to(beta, param_dtype) || !aligned4(dw) || !aligned4(db))
        return FF_ERR_ALIGN;
    if (rows > 0) {
        REFUSE(matrix_status(dy, dtype, lddy, n));
        REFUSE(ckpt_status(q, e));
    }
    hipStream_t s = (hipStream_t)stream;
    HIPCHK_T(FF_K_CKPT_DW, launch_ckpt_wgrad({dy, lddy, dtype, q, e, rows, n, k, gamma, beta, param_dtype, dw, db, accumulate, ws}, s));
    return FF_OK;
}

}  // extern "C"
