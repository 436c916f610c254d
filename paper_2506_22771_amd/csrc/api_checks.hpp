// Validation of arguments, on the host, that the calls on matrices of floating-point values share (api_norm.hip, api_blocks.hip).
#pragma once

#include "ff_internal.hpp"

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
