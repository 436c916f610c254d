// Group norm with an activation, backward: see group_norm.hpp.
#pragma once

#include "group_norm.hpp"

namespace ffi {

// ---- backward -----------------------------------------------------------------------------------------------------------
template <typename T> struct GnBackwardArgs {
    Slab s;
    const T* dy;          // may be null
    const T* x;           // or the checkpoint
    T* dx;                // may be null
    int64_t lddy, ldx, lddx;
    const float* coeff;   // may be null
    const float* mean;
    const float* rstd;
    const void* weight;
    const void* bias;
    CkptPtr k;
    float2* sums;         // [samples][channels], or [samples][blocks][channels]: sums of dz and dz h
    const float2* group;  // launch that applies: sums over groups of g and g h, by the group's size
    int32_t param_f32, blocks, rows;
    float inv_m;
};

// What a thread holds of one pixel.
template <typename T, bool FROM_X> struct GnPixel {
    Raw8<T> dy, x;
    u32x2 q;
    uint32_t e;
};
// Where a thread's chunks lie.
template <typename T, bool FROM_X> struct GnFrom {
    Walk<const T> dy, x;
    Walk<const int8_t> q;
    Walk<const uint8_t> e;
    __device__ __forceinline__ GnFrom(const GnBackwardArgs<T>& a, int64_t pixel0, int pl, int chunk, bool there)
        : dy(a.dy, a.lddy, pixel0, a.s.lanes, a.dy && there, pl, 8 * chunk), x(a.x, a.ldx, pixel0, a.s.lanes, FROM_X && there, pl, 8 * chunk),
          q(a.k.q, a.k.pitch, pixel0, a.s.lanes, !FROM_X && there, pl, 8 * chunk), e(a.k.e, a.k.epitch, pixel0, a.s.lanes, !FROM_X && there, pl, chunk >> 2) {}
    // the next pixel; n: columns of the chunk, 0 where there is no such pixel (the first one is read instead, and not used)
    template <bool RAGGED> __device__ __forceinline__ void load(const GnBackwardArgs<T>& a, GnPixel<T, FROM_X>& v, int n)
    {
        const int m = RAGGED ? n : 8;
        raw_zero(v.dy);
        if (a.dy) v.dy = load_raw(dy.here(n > 0), m);   // (uniform)
        dy.next();
        if constexpr (FROM_X) {
            v.x = load_raw(x.here(n > 0), m);
            x.next();
        } else {
            v.q = *(const u32x2*)q.here(n > 0);
            v.e = *e.here(n > 0);
            q.next();
            e.next();
        }
    }
};
// What a chunk's columns are scaled by.
template <typename T, bool FROM_X, int CELLS> struct GnGradChunk {
    float m[CELLS], rs[CELLS], w[8], b[8], c2;
};
template <typename T, bool FROM_X, int CELLS>
__device__ __forceinline__ void load_chunk(const GnBackwardArgs<T>& a, GnGradChunk<T, FROM_X, CELLS>& p, int64_t sample, int chunk, int n, int first, int group0, int groups)
{
    load_param<T>(a.weight, a.param_f32, 8 * (int64_t)chunk, n, 1.0f, p.w);
    load_param<T>(a.bias, a.param_f32, 8 * (int64_t)chunk, n, 0.0f, p.b);
    of_cells<CELLS>(first, a.s.d, groups, [&](int i, int g, int) {
        const int64_t from = sample * a.s.groups + (group0 + g);
        p.m[i] = FROM_X ? a.mean[from] : 0.0f;
        p.rs[i] = a.rstd[from];
    });
    p.c2 = a.coeff ? 2.0f * a.coeff[sample] : 0.0f;
}
template <typename T, bool FROM_X, int CELLS>
__device__ __forceinline__ void h_of(const GnPixel<T, FROM_X>& v, const GnGradChunk<T, FROM_X, CELLS>& p, float h[8])
{
    if constexpr (FROM_X) {
        raw_values(v.x, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = (h[i] - p.m[cell_of<CELLS>(i)]) * p.rs[cell_of<CELLS>(i)];
    } else {
        ckpt_values(v.q, v.e, h);
    }
}
// dz of one pixel.  (The identity without a goodness has f times c2 = 0 added: h is finite, or dz is NaN anyway.)
template <int ACT, typename T, bool FROM_X, int CELLS>
__device__ __forceinline__ void dz_of(const GnPixel<T, FROM_X>& v, const GnGradChunk<T, FROM_X, CELLS>& p, const float h[8], float dz[8])
{
    raw_values(v.dy, dz);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float f, d;
        act_of<T, ACT, true, false>(__builtin_fmaf(h[i], p.w[i], p.b[i]), f, d);
        dz[i] = __builtin_fmaf(p.c2, f, dz[i]) * d;
        if (i & 1) one_pixel_at_a_time();
    }
}
template <bool RAGGED> __device__ __forceinline__ void add_column_sums(const float h[8], const float dz[8], int n, float (&v)[2][8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool there = !RAGGED || i < n;
        v[0][i] = there ? v[0][i] + dz[i] : v[0][i];
        v[1][i] = there ? __builtin_fmaf(dz[i], h[i], v[1][i]) : v[1][i];
    }
}
template <typename T, bool RAGGED, bool FROM_X, int CELLS>
__device__ __forceinline__ void store_dx(T* to, int n, const float h[8], const float dz[8],
                                         const GnGradChunk<T, FROM_X, CELLS>& p, const float sg[CELLS], const float sh[CELLS])
{
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int k = cell_of<CELLS>(i);
        v[i] = p.rs[k] * __builtin_fmaf(-h[i], sh[k], p.w[i] * dz[i] - sg[k]);
    }
    store8(to, RAGGED ? n : 8, v);
}

// U: pixels of a thread
template <typename T, bool RAGGED, bool FROM_X, int CELLS, int ACT, int U> __global__ __launch_bounds__(1024, 4) void k_gn_backward(GnBackwardArgs<T> a)
{
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const Slab& s = a.s;
    const int item = item_of(s);
    if (item < 0) return;
    const int c = threadIdx.x % s.slots, pl = threadIdx.x / s.slots;
    const int sample = item / s.slices, slice = item - sample * s.slices, c0 = slice * s.slice;
    const int cols = min(s.slice, s.channels - c0), groups = max(1, cols / s.d);
    const int chunk = c0 / 8 + c, n = pl < s.lanes ? max(0, min(8, cols - 8 * c)) : 0;
    const int64_t pixel0 = (int64_t)sample * s.pixels;
    GnFrom<T, FROM_X> from(a, pixel0, pl, chunk, n > 0 && pl < s.pixels);
    GnPixel<T, FROM_X> px[U];
    GnGradChunk<T, FROM_X, CELLS> p;
    float v[2][8] = {};
#pragma unroll
    for (int u = 0; u < U; ++u) from.template load<RAGGED>(a, px[u], pl + u * s.lanes < s.pixels ? n : 0);
    load_chunk(a, p, sample, chunk, n, 8 * c, c0 / s.d, groups);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (n > 0 && pl + u * s.lanes < s.pixels) {
            float h[8], dz[8];
            h_of(px[u], p, h);
            dz_of<ACT>(px[u], p, h, dz);
            add_column_sums<RAGGED>(h, dz, n, v);
        }
        opaque(px[u].dy);
        if constexpr (FROM_X) opaque(px[u].x);
        else opaque(px[u].q);
        one_pixel_at_a_time();
    }
    const int cells = 8 * s.slots;
    float* const out = lds + 2 * cells * (1 + s.parts + s.lanes);
    float* const ws = out + 2 * ((cells + s.d - 1) / s.d + 1);
    if (pl == 0)
#pragma unroll
        for (int i = 0; i < 8; ++i) ws[8 * c + i] = p.w[i];
    sum_cells<2, 8>(v, s.slots, s.lanes, s.parts, c, pl, lds);
    if (a.sums)
        for (int t = threadIdx.x; t < cols; t += (int)blockDim.x) a.sums[(int64_t)sample * s.channels + c0 + t] = make_float2(lds[t], lds[cells + t]);
    if (a.dx) {
        sum_groups<2>(groups, s.d, out, [&](int k, int i) { return ws[i] * lds[k * cells + i]; });
        Walk<T> to(a.dx, a.lddx, pixel0, s.lanes, n > 0 && pl < s.pixels, pl, 8 * chunk);
        float sg[CELLS], sh[CELLS];
        of_cells<CELLS>(8 * c, s.d, groups, [&](int i, int g, int) {
            sg[i] = out[g] * a.inv_m;
            sh[i] = out[groups + g] * a.inv_m;
        });
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (n > 0 && pl + u * s.lanes < s.pixels) {
                float h[8], dz[8];
                h_of(px[u], p, h);
                dz_of<ACT>(px[u], p, h, dz);
                store_dx<T, RAGGED, FROM_X, CELLS>(to.p, n, h, dz, p, sg, sh);
            }
            to.next();
            one_pixel_at_a_time();
        }
    }
}

// Sums of columns over a block of pixels.
template <typename T, bool RAGGED, bool FROM_X, int CELLS, int ACT> __global__ __launch_bounds__(GN_SPLIT_THREADS, 4) void k_gn_backward_sums(GnBackwardArgs<T> a)
{
    constexpr int U = 2;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const Slab& s = a.s;
    const int item = item_of(s);
    if (item < 0) return;
    const int c = threadIdx.x % s.slots, pl = threadIdx.x / s.slots;
    const int sb = item / s.slices, sample = sb / a.blocks, slice = item - sb * s.slices, block = sb - sample * a.blocks;
    const int chunk = slice * s.slots + c, c0 = slice * s.slice, cols = min(s.slice, s.channels - c0);
    const int n = pl < s.lanes ? max(0, min(8, s.channels - 8 * chunk)) : 0;
    const int p0 = block * a.rows, pixels = min(a.rows, s.pixels - p0);
    const int64_t pixel0 = (int64_t)sample * s.pixels + p0;
    GnGradChunk<T, FROM_X, CELLS> p;
    load_chunk(a, p, sample, chunk, n, 8 * min(chunk, (s.channels - 1) / 8), 0, s.groups);
    float v[2][8] = {};
    for (int first = 0; first < pixels; first += U * s.lanes) {
        GnFrom<T, FROM_X> from(a, pixel0, first + pl, chunk, n > 0 && first + pl < pixels);
        GnPixel<T, FROM_X> px[U];
#pragma unroll
        for (int u = 0; u < U; ++u) from.template load<RAGGED>(a, px[u], first + pl + u * s.lanes < pixels ? n : 0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (n > 0 && first + pl + u * s.lanes < pixels) {
                float h[8], dz[8];
                h_of(px[u], p, h);
                dz_of<ACT>(px[u], p, h, dz);
                add_column_sums<RAGGED>(h, dz, n, v);
            }
            one_pixel_at_a_time();
        }
    }
    sum_cells<2, 8>(v, s.slots, s.lanes, s.parts, c, pl, lds);
    for (int t = threadIdx.x; t < cols; t += (int)blockDim.x) a.sums[(int64_t)sb * s.channels + c0 + t] = make_float2(lds[t], lds[8 * s.slots + t]);
}

// Sums of a sample's blocks: sums of its columns, and those of its groups by a group's size.  A workgroup takes `many` groups of up to 64 columns together, or one
// in tiles of 64 columns, sixteen threads to a column (4 x 256x256 x 64 fp16, 128 blocks: 4 us; one thread to a column 33).
template <typename T>
__global__ __launch_bounds__(1024) void k_gn_backward_join(const float2* part, float2* sums, float2* group, const void* weight, int param_f32, int64_t items,
                                                           int32_t per_sample, int32_t groups, int32_t d, int32_t many, int32_t blocks, float inv_m)
{
    __shared__ float2 red[16][64];
    const int col = threadIdx.x & 63, lane = threadIdx.x >> 6, channels = groups * d;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t sample = item / per_sample;
        const int g0 = (int)(item - sample * per_sample) * many, here = min(many, groups - g0), c0 = g0 * d, cols = here * d;
        float2 of_group = make_float2(0, 0);
        for (int first = 0; first < cols; first += 64) {
            const int c = first + col;
            float2 t = make_float2(0, 0);
            if (c < cols)
#pragma unroll 4
                for (int b = lane; b < blocks; b += 16) {
                    const float2 v = part[(sample * blocks + b) * channels + c0 + c];
                    t.x += v.x;
                    t.y += v.y;
                }
            __syncthreads();   // (what the last tile left in red has been read)
            red[lane][col] = t;
            __syncthreads();
            if (lane == 0) {
                for (int l = 1; l < 16; ++l) {
                    t.x += red[l][col].x;
                    t.y += red[l][col].y;
                }
                float w[8] = {};
                if (c < cols) {
                    sums[sample * channels + c0 + c] = t;
                    load_param<T>(weight, param_f32, c0 + c, 1, 1.0f, w);
                }
                t = make_float2(w[0] * t.x, w[0] * t.y);   // (zero behind the last column)
                if (here > 1) {
                    red[0][col] = t;
                } else {
                    of_group.x += wave_sum(t.x);
                    of_group.y += wave_sum(t.y);
                }
            }
        }
        if (here > 1) {
            __syncthreads();
            for (int g = threadIdx.x; g < here; g += 1024) {
                for (int i = 0; i < d; ++i) {
                    of_group.x += red[0][g * d + i].x;
                    of_group.y += red[0][g * d + i].y;
                }
                group[sample * groups + g0 + g] = make_float2(of_group.x * inv_m, of_group.y * inv_m);
                of_group = make_float2(0, 0);
            }
        } else if (threadIdx.x == 0) {
            group[sample * groups + g0] = make_float2(of_group.x * inv_m, of_group.y * inv_m);
        }
    }
}

template <typename T, bool RAGGED, bool FROM_X, int CELLS, int ACT> __global__ __launch_bounds__(GN_SPLIT_THREADS, 4) void k_gn_backward_apply(GnBackwardArgs<T> a)
{
    const Slab& s = a.s;
    const int item = item_of(s);
    if (item < 0) return;
    const int c = threadIdx.x % s.slots, pl = threadIdx.x / s.slots;
    const int sb = item / s.slices, sample = sb / a.blocks, slice = item - sb * s.slices, block = sb - sample * a.blocks;
    const int chunk = slice * s.slots + c, n = pl < s.lanes ? max(0, min(8, s.channels - 8 * chunk)) : 0;
    const int p0 = block * a.rows, pixels = min(a.rows, s.pixels - p0);
    const int64_t pixel0 = (int64_t)sample * s.pixels + p0;
    GnFrom<T, FROM_X> from(a, pixel0, pl, chunk, n > 0 && pl < pixels);
    GnPixel<T, FROM_X> px[GN_APPLY_ROWS];
#pragma unroll
    for (int u = 0; u < GN_APPLY_ROWS; ++u) from.template load<RAGGED>(a, px[u], pl + u * s.lanes < pixels ? n : 0);
    const int first = 8 * min(chunk, (s.channels - 1) / 8);
    GnGradChunk<T, FROM_X, CELLS> p;
    load_chunk(a, p, sample, chunk, n, first, 0, s.groups);
    Walk<T> to(a.dx, a.lddx, pixel0, s.lanes, n > 0 && pl < pixels, pl, 8 * chunk);
    float sg[CELLS], sh[CELLS];
    of_cells<CELLS>(first, s.d, s.groups, [&](int i, int g, int) {
        const float2 t = a.group[(int64_t)sample * s.groups + g];
        sg[i] = t.x;
        sh[i] = t.y;
    });
#pragma unroll
    for (int u = 0; u < GN_APPLY_ROWS; ++u) {
        if (n > 0 && pl + u * s.lanes < pixels) {
            float h[8], dz[8];
            h_of(px[u], p, h);
            dz_of<ACT>(px[u], p, h, dz);
            store_dx<T, RAGGED, FROM_X, CELLS>(to.p, n, h, dz, p, sg, sh);
        }
        to.next();
        one_pixel_at_a_time();
    }
}

// ---- launches ----------------------------------------------------------------------------------------------------
template <typename T, bool RAGGED, bool FROM_X, int CELLS, int ACT> static hipError_t gn_backward_of(const GroupNormBackwardLaunch& g, hipStream_t s)
{
    GnBackwardArgs<T> a = {};
    const int64_t d = g.channels / g.groups;
    const GnPlan p = gn_plan(g.samples, g.pixels, g.channels, g.groups, sizeof(T), false, g.channels, true);
    a.dy = (const T*)g.dy;
    a.x = (const T*)g.x;
    a.dx = (T*)g.dx;
    a.lddy = g.lddy;
    a.ldx = g.ldx;
    a.lddx = g.lddx;
    a.coeff = g.coeff;
    a.mean = g.mean;
    a.rstd = g.rstd;
    a.weight = g.weight;
    a.bias = g.bias;
    a.param_f32 = g.param_dtype == FF_F32;
    a.inv_m = (float)(1.0 / ((double)g.pixels * (double)d));
    if (!FROM_X) a.k = ckpt_ptr(g.q, g.e, g.channels);
    float2* const sums = (float2*)g.ws;   // of every sample's columns
    if (p.whole) {
        a.sums = g.dweight || g.dbias ? sums : nullptr;
        a.s = slab_of(p.cut, g.samples, g.pixels, g.channels, g.groups, 1, 8);
        const size_t lds = gn_lds(p.cut.threads, p.cut.slots, 8, d);
        // slabs of a quarter of the pixels by a kernel of no more (45 x 33x33 x 1 bf16 forward 14.0 us, by the other 18.7; 138 x 5x5 x 23 backward 10.0 and 12.1)
        constexpr int U = gn_rows(sizeof(T), true), FEW = U / 4;
        auto* const kernel = p.cut.lanes * FEW >= g.pixels ? k_gn_backward<T, RAGGED, FROM_X, CELLS, ACT, FEW> : k_gn_backward<T, RAGGED, FROM_X, CELLS, ACT, U>;
        GN_TRY(with_lds(kernel, lds));
        GN_TRY(launch_items(a, [&](unsigned grid, const auto& part) { kernel<<<grid, p.cut.threads, lds, s>>>(part); }));
    } else {
        float2* const part = sums + g.samples * g.channels;
        float2* const group = part + g.samples * g.channels * p.blocks;
        a.sums = part;
        a.blocks = p.blocks;
        a.rows = (int32_t)((g.pixels + p.blocks - 1) / p.blocks);
        a.s = slab_of(p.stat, g.samples, g.pixels, g.channels, g.groups, p.blocks, 8);
        const size_t lds = gn_lds(p.stat.threads, p.stat.slots, 8, d);
        GN_TRY(launch_items(a, [&](unsigned grid, const auto& part) { k_gn_backward_sums<T, RAGGED, FROM_X, CELLS, ACT><<<grid, GN_SPLIT_THREADS, lds, s>>>(part); }));
        const int64_t many = std::max<int64_t>(1, std::min(g.groups, 64 / d)), per_sample = (g.groups + many - 1) / many, items = g.samples * per_sample;
        k_gn_backward_join<T><<<(unsigned)std::min<int64_t>(items, GN_MOST_GRID), 1024, 0, s>>>(part, sums, group, g.weight, a.param_f32, items, (int32_t)per_sample,
                                                                                       (int32_t)g.groups, (int32_t)d, (int32_t)many, p.blocks, a.inv_m);
        GN_TRY(hipGetLastError());
        if (g.dx) {
            a.group = group;
            a.blocks = p.apply_blocks;
            a.rows = p.cut.lanes * GN_APPLY_ROWS;
            a.s = slab_of(p.cut, g.samples, g.pixels, g.channels, g.groups, p.apply_blocks, 8);
            GN_TRY(launch_items(a, [&](unsigned grid, const auto& part) { k_gn_backward_apply<T, RAGGED, FROM_X, CELLS, ACT><<<grid, GN_SPLIT_THREADS, 0, s>>>(part); }));
        }
    }
    return launch_gn_params(sums, g, s);
}
template <typename T> hipError_t gn_backward_typed(const GroupNormBackwardLaunch& g, hipStream_t s)
{
    return by_columns(g.channels, g.groups, [&](auto ragged, auto cells) {
        return by_activation(g.act, [&](auto act) {
            constexpr bool RAGGED = decltype(ragged)::value;
            constexpr int CELLS = decltype(cells)::value, ACT = decltype(act)::value;
            return g.x ? gn_backward_of<T, RAGGED, true, CELLS, ACT>(g, s) : gn_backward_of<T, RAGGED, false, CELLS, ACT>(g, s);
        });
    });
}

}  // namespace ffi
