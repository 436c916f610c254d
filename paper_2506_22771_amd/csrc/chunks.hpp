// Launches over all chunks of a matrix, in order: what the checkpoints (ckpt.hip), the gated layer's gradient (gated_grad.hip) and dropout (dropout.hip) share.
#pragma once

#include <type_traits>

#include "ckpt.hpp"

namespace ffi {

constexpr int CK_THREADS = 256;

// Consecutive chunks of a matrix; rows are `slots` chunks long (a multiple of four, so that quads hold blocks).
struct Chunks {
    int64_t total;
    uint32_t slots, magic;   // magic: ceil(2^32 / slots)
};
static Chunks chunks_of(int64_t rows, int64_t bytes_or_cols)
{
    const int64_t slots = (bytes_or_cols + 31) / 32 * 4;
    return {rows * slots, (uint32_t)slots, (uint32_t)(((uint64_t(1) << 32) + (uint64_t)slots - 1) / (uint64_t)slots)};
}
// Row (from the workgroup's first one, row0, on) and chunk of `at` chunks (fewer than 4096) behind the workgroup's first one, (row0, chunk0).  Rows of 4096
// chunks or more: at most one row further; shorter ones: at + chunk0 < 8192, where the product with the rounded-up reciprocal has the quotient exactly.
__device__ __forceinline__ void chunk_place(const Chunks& c, uint32_t chunk0, uint32_t at, uint32_t& r, uint32_t& chunk)
{
    const uint32_t o = chunk0 + at;
    r = c.slots >= 4096u ? (o >= c.slots ? 1u : 0u) : __umulhi(o, c.magic);
    chunk = o - r * c.slots;
}
__device__ __forceinline__ void chunk_first(const Chunks& c, int64_t first, int64_t& row0, uint32_t& chunk0)
{
    const uint32_t r = (uint32_t)first / c.slots;   // (a matrix has fewer than 2^31 chunks: size_status)
    row0 = r;
    chunk0 = (uint32_t)first - r * c.slots;
}

// A chunk `at` chunks behind the workgroup's first one: its place (the workgroup's first row's first chunk where there is none) and how many of its columns
// exist.
__device__ __forceinline__ int chunk_at(const Chunks& c, int cols, int64_t first, uint32_t chunk0, uint32_t at, uint32_t& r, uint32_t& chunk)
{
    chunk_place(c, chunk0, at, r, chunk);
    const bool there = first + at < c.total;
    r = there ? r : 0;
    chunk = there ? chunk : 0;
    return there ? max(0, min(8, cols - 8 * (int)chunk)) : 0;
}

template <typename F> static void by_ends(int64_t cols, bool in_place, F&& launch)
{
    if (cols % 8 == 0) launch(std::integral_constant<RowEnds, ROWS_WHOLE>());
    else if (cols > 8 && !in_place) launch(std::integral_constant<RowEnds, ROWS_RAGGED>());
    else launch(std::integral_constant<RowEnds, ROWS_OWN>());
}
template <int U> static unsigned ckpt_grid(const Chunks& c) { return (unsigned)((c.total + CK_THREADS * U - 1) / (CK_THREADS * U)); }

}  // namespace ffi
