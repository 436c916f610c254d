// Group norm with an activation over channels-last maps, forward and backward.
//
//   per sample and group, over its d channels at all P pixels:  mean, rstd = 1 / sqrt(1/(P d) sum (x - mean)^2 + eps),  h = (x - mean) rstd
//   z = h gamma + beta,  y = f(z),  G = sum over the sample of f(z)^2
//   dz = (dy + 2 c f(z)) f'(z),  dgamma = sum over pixels and samples of dz h,  dbeta = sum of dz
//   dx = rstd (g - 1/(P d) sum over the group of g - h 1/(P d) sum over the group of g h),  g = gamma dz
//
// Statistics, products and sums are fp32 (the means of parts of a group, and dgamma and dbeta over the samples, are joined in 64 bits); y and dx are rounded once.  As in the layer norm, the mean of
// the deviations is taken out of groups farther from zero than they are wide (norm_math.hpp).
//
// Memory bounds all of it.  A workgroup's threads lie over a slab of whole groups: a chunk of eight columns is a thread's own from pixel to pixel, so that
// parameters and sums of columns stay in registers, and sums meet in LDS once.  Where such a slab fits the registers of a workgroup, everything is read once
// (one launch, `whole` below; group_norm_plan.hpp).  Else a first launch sums parts of groups, a small one joins them, and a third reads again and applies.
// The sums of all samples, dgamma and dbeta, are a launch of their own over sums of columns per sample.
//
// Measured, 512 x 32x32 x 128 bf16 in 32 groups, SiLU: forward 62 us (4.3 TB/s), with codes to nearest 103, stochastic 114 to 118 (41 vector instructions a value,
// 77 us of issue); backward from x 119, from codes 107 to 112 (40 a value, four of them transcendental, in quarter time); identity 58, 93, 104, 104 and 93.  fp32 at the
// same size 135 (4.0 TB/s), 153, 160, 190 and 167.  Split: 8 x 113x113 x 120 fp32 GELU 35 us forward (statistics 12, join 4, apply 20) and 56 backward; 4 x 256x256 x
// 64 fp16 SiLU 31 and 45.  Latency: 1 x 32x32 x 128 bf16 10 us, 512 x 4x4 x 512 fp32 12 forward and 19 backward.
#pragma once

#include "act.hpp"
#include "blocks.hpp"
#include "group_norm_plan.hpp"
#include "norm_math.hpp"

namespace ffi {

// ---- slabs ------------------------------------------------------------------------------------------------------------
struct Slab {
    int32_t slots, lanes, slice, slices;   // see GnCut
    int32_t pixels, channels, groups, d;
    int32_t parts;             // threads that share the sum of a cell over the lanes, at most
    int32_t first, items, per_xcd;   // workgroups' work, (sample, [block of pixels,] slice): this launch's.  (Fewer than there are chunks, which are fewer than 2^31.)
};
// A workgroup's item, or -1.  Items in turn to the eight XCDs, so that neighbours, which share cache lines, meet in one L2.
__device__ __forceinline__ int item_of(const Slab& s)
{
    const int i = (int)(blockIdx.x & 7) * s.per_xcd + (int)(blockIdx.x >> 3);
    return i < s.items ? s.first + i : -1;
}

// A thread's way through a matrix, from its chunk of its first pixel on.  (Step by step: products of the scalar step with every pixel's number are more scalars
// than there are, and reading what was spilled of them took a tenth of all instructions.)
template <typename P> struct Walk {
    P *p, *first;
    int64_t step;
    __device__ __forceinline__ Walk(P* matrix, int64_t ld, int64_t pixel0, int lanes, bool there, int pl, int at)
        : p(there ? element(matrix + pixel0 * ld, ld, 0, pl, at) : matrix + pixel0 * ld), first(p), step((int64_t)lanes * ld) {}
    __device__ __forceinline__ void next() { p += step; }
    __device__ __forceinline__ P* here(bool there) const { return there ? p : first; }   // a pixel that is not there: the first
};

// What the compiler is not to mix with what follows: several pixels' values at once take more registers than there are.
__device__ __forceinline__ void one_pixel_at_a_time() { __builtin_amdgcn_sched_barrier(0); }

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// What a thread keeps apart of its chunk: the halves (CELLS 2), where every group is a multiple of four channels, or every column (8).
template <int CELLS> constexpr int cell_of(int column) { return CELLS == 2 ? column >> 2 : column; }
// Every cell's group, counted from the slice's first column on, and its first column's place in it.
template <int CELLS, typename F> __device__ __forceinline__ void of_cells(int first, int d, int groups, F&& each)
{
    if constexpr (CELLS == 2) {
        const int g0 = first / d, g1 = (first + 4) / d;
        each(0, min(g0, groups - 1), first - g0 * d);
        each(1, min(g1, groups - 1), first + 4 - g1 * d);
    } else {
        int g = first / d, at = first - g * d;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            each(i, min(g, groups - 1), at);
            if (++at == d) {
                at = 0;
                ++g;
            }
        }
    }
}

// Sums over the lanes of K values of every cell, into lds[k * cells + i], cell i of the slots * CELLS.  lds: K cells (1 + parts + lanes) floats.  A barrier ends it.
template <int K, int CELLS> __device__ __forceinline__ float* place_cells(const float (&v)[K][CELLS], int slots, int lanes, int most_parts, int c, int pl, float* lds)
{
    const int cells = slots * CELLS;
    float* const all = lds + K * cells * (1 + most_parts);
    if (pl < lanes) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < CELLS; ++i) all[(k * lanes + pl) * cells + c * CELLS + i] = v[k][i];
    }
    __syncthreads();
    return all;
}
template <int K, int CELLS>
__device__ __forceinline__ void sum_cells(const float (&v)[K][CELLS], int slots, int lanes, int most_parts, int c, int pl, float* lds)
{
    const int cells = slots * CELLS, parts = max(1, min(most_parts, (int)blockDim.x / (K * cells)));
    const float* const all = place_cells(v, slots, lanes, most_parts, c, pl, lds);
    float* const some = parts > 1 ? lds + K * cells : lds;
    for (int t = threadIdx.x; t < K * cells * parts; t += (int)blockDim.x) {
        const int part = t / (K * cells), kc = t - part * (K * cells), k = K > 1 && kc >= cells ? 1 : 0, i = kc - k * cells;
        float s = 0;
#pragma unroll 4
        for (int l = part; l < lanes; l += parts) s += all[(k * lanes + l) * cells + i];
        some[t] = s;
    }
    __syncthreads();
    if (parts == 1) return;
    for (int t = threadIdx.x; t < K * cells; t += (int)blockDim.x) {
        float s = 0;
#pragma unroll 4
        for (int part = 0; part < parts; ++part) s += some[part * (K * cells) + t];
        lds[t] = s;
    }
    __syncthreads();
}
// Sums over the `n` cells of each of `groups` groups, by value(k, cell), into out[k * groups + g].  A barrier ends it.
template <int K, typename F> __device__ __forceinline__ void sum_groups(int groups, int n, float* out, F&& value)
{
    if (n <= 16) {
        for (int t = threadIdx.x; t < K * groups; t += (int)blockDim.x) {
            const int k = K > 1 && t >= groups ? 1 : 0, g = t - k * groups;
            float s = 0;
            for (int i = 0; i < n; ++i) s += value(k, g * n + i);
            out[t] = s;
        }
    } else {
        for (int t = threadIdx.x >> 6; t < K * groups; t += (int)blockDim.x / 64) {
            const int k = K > 1 && t >= groups ? 1 : 0, g = t - k * groups;
            float s = 0;
            for (int i = threadIdx.x & 63; i < n; i += 64) s += value(k, g * n + i);
            s = wave_sum(s);
            if ((threadIdx.x & 63) == 0) out[t] = s;
        }
    }
    __syncthreads();
}
// Both at once, for sums of cells that nobody else asks for: out[k * groups + g], K up to 2.  A barrier ends it.
template <int K, int CELLS>
__device__ __forceinline__ void sum_lanes_of_groups(const float (&v)[K][CELLS], int slots, int lanes, int most_parts, int c, int pl, int groups, int n, float* lds, float* out)
{
    const int cells = slots * CELLS;
    if (lanes * n <= 16) {   // few values to a group: one step, a thread each
        const float* const all = place_cells(v, slots, lanes, most_parts, c, pl, lds);
        for (int t = threadIdx.x; t < K * groups; t += (int)blockDim.x) {
            const int k = K > 1 && t >= groups ? 1 : 0, g = t - k * groups;
            float s = 0;
            for (int l = 0; l < lanes; ++l)
                for (int i = 0; i < n; ++i) s += all[(k * lanes + l) * cells + g * n + i];
            out[t] = s;
        }
        __syncthreads();
    } else {
        sum_cells<K, CELLS>(v, slots, lanes, most_parts, c, pl, lds);
        sum_groups<K>(groups, n, out, [&](int k, int i) { return lds[k * cells + i]; });
    }
}

// Sum of a workgroup's values, in thread 0.  red: a word per wavefront.  A barrier begins it.
__device__ __forceinline__ float sum_block(float v, float* red)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0;
    if (threadIdx.x == 0)
        for (int w = 0; w < (int)blockDim.x / 64; ++w) s += red[w];
    return s;
}

// ---- launches ----------------------------------------------------------------------------------------------------
static Slab slab_of(const GnCut& c, int64_t samples, int64_t pixels, int64_t channels, int64_t groups, int64_t blocks, int cells)
{
    Slab s = {};
    s.slots = c.slots;
    s.lanes = c.lanes;
    s.slice = c.slice;
    s.slices = c.slices;
    s.pixels = (int32_t)pixels;
    s.channels = (int32_t)channels;
    s.groups = (int32_t)groups;
    s.d = (int32_t)(channels / groups);
    s.parts = gn_parts(c.threads, c.slots, cells);
    s.items = (int32_t)(samples * blocks * c.slices);
    return s;
}
// A launch has fewer than 2^32 threads: one after the other for more items than that.
template <typename Args, typename F> static hipError_t launch_items(Args a, F&& launch)
{
    const int64_t all = a.s.items;
    for (int64_t first = 0; first < all; first += GN_MOST_GRID) {
        a.s.first = (int32_t)first;
        a.s.items = (int32_t)std::min<int64_t>(all - first, GN_MOST_GRID);
        a.s.per_xcd = (a.s.items + 7) / 8;
        launch((unsigned)(8 * a.s.per_xcd), a);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

// LDS for a kernel's launch.  The plan asks for no more than there is; an error of the runtime is returned here and not kept for the next call to find.
template <typename F> static hipError_t with_lds(F* kernel, size_t bytes)
{
    if (bytes <= 65536) return hipSuccess;
    if (bytes > GN_MOST_LDS) return hipErrorInvalidValue;
    const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != hipSuccess) (void)hipGetLastError();
    return e;
}
#define GN_TRY(e) do { const hipError_t _e = (e); if (_e != hipSuccess) return _e; } while (0)

template <int CELLS> using Cells = std::integral_constant<int, CELLS>;
// Rows of whole chunks whose halves lie in one group each; of whole chunks; any.
template <typename F> static hipError_t by_columns(int64_t channels, int64_t groups, F&& launch)
{
    using Whole = std::false_type;
    using Ragged = std::true_type;
    if (channels % 8 != 0) return launch(Ragged(), Cells<8>());
    return gn_cells(channels, channels / groups, false) == 2 ? launch(Whole(), Cells<2>()) : launch(Whole(), Cells<8>());
}
template <typename F> static hipError_t by_activation(int act, F&& launch)
{
    switch (act) {
        case FF_ACT_RELU: return launch(std::integral_constant<int, FF_ACT_RELU>());
        case FF_ACT_GELU: return launch(std::integral_constant<int, FF_ACT_GELU>());
        case FF_ACT_SILU: return launch(std::integral_constant<int, FF_ACT_SILU>());
        default: return launch(std::integral_constant<int, FF_ACT_IDENTITY>());
    }
}

// group_norm.hip
hipError_t launch_gn_join(const float4* part, float4* stats, const GroupNormForwardLaunch& f, int32_t parts, hipStream_t s);
hipError_t launch_gn_goodness(const float* part, float* goodness, int64_t samples, int64_t parts, hipStream_t s);
hipError_t launch_gn_params(const float2* sums, const GroupNormBackwardLaunch& g, hipStream_t s);
// of one element type: group_norm_{f32,bf16,f16}.hip
template <typename T> hipError_t gn_forward_typed(const GroupNormForwardLaunch& f, hipStream_t s);
template <typename T> hipError_t gn_backward_typed(const GroupNormBackwardLaunch& g, hipStream_t s);

}  // namespace ffi
