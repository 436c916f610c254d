// Group norm with an activation, forward: see group_norm.hpp.
#include "group_norm.hpp"

namespace ffi {

// ---- forward ------------------------------------------------------------------------------------------------------------
template <typename T> struct GnForwardArgs {
    Slab s;
    const T* x;
    T* y;
    int64_t ldx, ldy;
    const void* weight;
    const void* bias;
    float* mean;
    float* rstd;
    float* good;       // partial sums of the goodness, or null
    float4* part;      // statistics' launch: mean, rest of the mean, squared deviations, values, of every part of a group
    const float4* stats;   // launch that applies: mean, its rest, rstd
    CkptPtr k;
    CkptRound r;
    int32_t act, param_f32, pieces, blocks, rows;   // rows: pixels of a workgroup
    float eps, inv_m;
};

// What a chunk's columns are normalised and scaled by.  An fp32 group's mean has a second word, what its rounding left of it; of 16-bit values that is
// below their own rounding.
template <typename T, int CELLS> struct GnChunk {
    float m[CELLS], rest[sizeof(T) == 4 ? CELLS : 1], rs[CELLS], w[8], b[8];
    __device__ __forceinline__ void mean(int i, float hi, float lo)
    {
        if constexpr (sizeof(T) == 4) {
            m[i] = hi;
            rest[i] = lo;
        } else {
            m[i] = hi + lo;
        }
    }
    __device__ __forceinline__ float h(float x, int i) const
    {
        float v = x - m[cell_of<CELLS>(i)];
        if constexpr (sizeof(T) == 4) v -= rest[cell_of<CELLS>(i)];
        return v * rs[cell_of<CELLS>(i)];
    }
};

// One chunk: normalised, kept, activated, stored; the sum of its squares.  n of its columns exist (none: its share of the codes' pad is written).
template <typename T, bool RAGGED, bool KEPT, int CELLS>
__device__ __forceinline__ float finish_chunk(const GnForwardArgs<T>& a, const Raw8<T>& raw, int64_t pixel, int chunk, int slots, int n, const GnChunk<T, CELLS>& p)
{
    float v[8], f[8];
    raw_values(raw, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p.h(v[i], i);
    if (RAGGED)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? v[i] : 0.0f;
    if constexpr (KEPT) {
        const uint32_t top = quad_max_u32(n > 0 ? abs_max_bits(v) : 0u), e = ckpt_exponent(top);
        const u32x2 q = ckpt_codes(v, top, e, a.r, (uint64_t)pixel * (uint32_t)a.s.channels + 8 * (uint32_t)chunk);
        ckpt_store_chunk(a.k, a.k.q + pixel * a.k.pitch, a.k.e + pixel * a.k.epitch, chunk, slots, n > 0, q, e);
    }
    if (n <= 0) return 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_fmaf(v[i], p.w[i], p.b[i]);
    activate<T>(a.act, v, f);
    store8(a.y + (pixel * a.ldy + 8 * chunk), RAGGED ? n : 8, f);
    float s = 0;
    if (a.good)   // (uniform)
#pragma unroll
        for (int i = 0; i < 8; ++i) s = !RAGGED || i < n ? __builtin_fmaf(f[i], f[i], s) : s;
    return s;
}

template <typename T, bool RAGGED, bool KEPT, int CELLS> __global__ __launch_bounds__(1024, 4) void k_gn_forward(GnForwardArgs<T> a)
{
    constexpr int U = gn_rows(sizeof(T), false);
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const Slab& s = a.s;
    const int row_slots = KEPT ? (int)((a.k.pitch + 31) / 32 * 4) : (s.channels + 7) / 8;
    for (int64_t turn = blockIdx.x; turn < 8 * s.per_xcd; turn += gridDim.x) {
        const int64_t item = item_of(s, turn);
        if (item < 0) continue;
        int c, pl;
        place_of(s, c, pl);
        const int64_t sample = item / s.slices;
        const int slice = (int)(item - sample * s.slices), c0 = slice * s.slice;
        const int cols = min(s.slice, s.channels - c0), groups = max(1, cols / s.d);
        const int chunk = c0 / 8 + c, n = pl < s.lanes ? max(0, min(8, cols - 8 * c)) : 0;
        const bool live = pl < s.lanes && chunk < row_slots;
        const int64_t pixel0 = sample * s.pixels;
        // a chunk that does not exist is read from a place that does, and not used
        const T* const x0 = a.x + pixel0 * a.ldx;
        const T* const x1 = n > 0 && pl < s.pixels ? element(x0, a.ldx, 0, pl, 8 * chunk) : x0;
        const int64_t step = (int64_t)s.lanes * a.ldx;
        Raw8<T> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool there = n > 0 && pl + u * s.lanes < s.pixels;
            raw[u] = load_raw(x1 + (there ? u * step : 0), RAGGED ? (there ? n : 0) : 8);
        }
        float v[1][CELLS] = {}, v2[2][CELLS] = {}, m[CELLS];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (n > 0 && pl + u * s.lanes < s.pixels) {
                float t[8];
                raw_values(raw[u], t);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[0][cell_of<CELLS>(i)] += t[i];
            }
            opaque(raw[u]);
            one_pixel_at_a_time();
        }
        const int per_group = s.d * CELLS / 8;
        float* const out = lds + 2 * s.slots * CELLS * (1 + s.parts + s.lanes);
        sum_cells<1, CELLS>(v, s.slots, s.lanes, s.parts, c, pl, lds);
        sum_groups<1>(groups, per_group, out, [&](int, int i) { return lds[i]; });
        of_cells<CELLS>(8 * c, s.d, groups, [&](int i, int g, int) { m[i] = out[g] * a.inv_m; });
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (n > 0 && pl + u * s.lanes < s.pixels) {
                float t[8];
                raw_values(raw[u], t);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float dev = !RAGGED || i < n ? t[i] - m[cell_of<CELLS>(i)] : 0.0f;
                    v2[0][cell_of<CELLS>(i)] += dev;
                    v2[1][cell_of<CELLS>(i)] = __builtin_fmaf(dev, dev, v2[1][cell_of<CELLS>(i)]);
                }
            }
            opaque(raw[u]);
            one_pixel_at_a_time();
        }
        const int cells = s.slots * CELLS;
        sum_cells<2, CELLS>(v2, s.slots, s.lanes, s.parts, c, pl, lds);
        GnChunk<T, CELLS> p;
        load_param<T>(a.weight, a.param_f32, 8 * (int64_t)chunk, n, 1.0f, p.w);
        load_param<T>(a.bias, a.param_f32, 8 * (int64_t)chunk, n, 0.0f, p.b);
        sum_groups<2>(groups, per_group, out, [&](int k, int i) { return lds[k * cells + i]; });
        of_cells<CELLS>(8 * c, s.d, groups, [&](int i, int g, int at) {
            const float square = out[groups + g] * a.inv_m, rest = mean_rest(m[i], out[g] * a.inv_m, square);
            p.mean(i, m[i], rest);
            p.rs[i] = inverse_root(variance(square, rest) + a.eps);
            if (pl == 0 && at == 0 && i * (8 / CELLS) < n) {
                const int64_t to = sample * s.groups + (c0 / s.d + g);
                if (a.mean) a.mean[to] = m[i] + rest;
                if (a.rstd) a.rstd[to] = p.rs[i];
            }
        });
        float good = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = pl + u * s.lanes;
            if (live && at < s.pixels) good += finish_chunk<T, RAGGED, KEPT, CELLS>(a, raw[u], pixel0 + at, chunk, row_slots, n, p);
            one_pixel_at_a_time();
        }
        if (a.good) {
            good = sum_block(good, lds);
            if (threadIdx.x == 0) a.good[item] = good;
        }
        __syncthreads();   // (the next item's sums go where this one's lie)
    }
}

// Statistics of parts of groups: a block of pixels of a slice, which is of whole groups or a piece of one.
template <typename T, bool RAGGED, int CELLS> __global__ __launch_bounds__(GN_SPLIT_THREADS, 4) void k_gn_stats(GnForwardArgs<T> a)
{
    constexpr int U = GN_STAT_ROWS;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const Slab& s = a.s;
    for (int64_t turn = blockIdx.x; turn < 8 * s.per_xcd; turn += gridDim.x) {
        const int64_t item = item_of(s, turn);
        if (item < 0) continue;
        int c, pl;
        place_of(s, c, pl);
        const int64_t sb = item / s.slices, sample = sb / a.blocks;
        const int slice = (int)(item - sb * s.slices), block = (int)(sb - sample * a.blocks);
        // the slice's columns and first group
        const bool one = a.pieces > 1;   // the slice lies in one group
        const int group0 = one ? slice / a.pieces : slice * (s.slice / s.d), piece = one ? slice - group0 * a.pieces : 0;
        const int c0 = group0 * s.d + piece * s.slice;
        const int cols = one ? min(s.slice, s.d - piece * s.slice) : min(s.slice, s.channels - c0);
        const int groups = one ? 1 : cols / s.d;
        const int n = pl < s.lanes ? max(0, min(8, cols - 8 * c)) : 0;
        const int p0 = block * a.rows, pixels = min(a.rows, s.pixels - p0);
        const T* const x0 = a.x + (sample * s.pixels + p0) * a.ldx + c0;
        const T* const x1 = n > 0 && pl < pixels ? element(x0, a.ldx, 0, pl, 8 * c) : x0;
        const int64_t step = (int64_t)s.lanes * a.ldx;
        Raw8<T> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool there = n > 0 && pl + u * s.lanes < pixels;
            raw[u] = load_raw(x1 + (there ? u * step : 0), RAGGED ? (there ? n : 0) : 8);
        }
        float v[1][CELLS] = {}, v2[2][CELLS] = {}, m[CELLS];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (n > 0 && pl + u * s.lanes < pixels) {
                float t[8];
                raw_values(raw[u], t);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[0][cell_of<CELLS>(i)] += t[i];
            }
            opaque(raw[u]);
            one_pixel_at_a_time();
        }
        const int cells = s.slots * CELLS, per_group = one ? cells : s.d * CELLS / 8, d = one ? 8 * s.slots : s.d;
        const float count = (float)(pixels * (one ? cols : s.d)), inv = 1.0f / count;
        float* const out = lds + 2 * cells * (1 + s.parts + s.lanes);
        sum_cells<1, CELLS>(v, s.slots, s.lanes, s.parts, c, pl, lds);
        sum_groups<1>(groups, per_group, out, [&](int, int i) { return lds[i]; });
        of_cells<CELLS>(8 * c, d, groups, [&](int i, int g, int) { m[i] = out[g] * inv; });
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (n > 0 && pl + u * s.lanes < pixels) {
                float t[8];
                raw_values(raw[u], t);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float dev = !RAGGED || i < n ? t[i] - m[cell_of<CELLS>(i)] : 0.0f;
                    v2[0][cell_of<CELLS>(i)] += dev;
                    v2[1][cell_of<CELLS>(i)] = __builtin_fmaf(dev, dev, v2[1][cell_of<CELLS>(i)]);
                }
            }
        }
        sum_cells<2, CELLS>(v2, s.slots, s.lanes, s.parts, c, pl, lds);
        sum_groups<2>(groups, per_group, out, [&](int k, int i) { return lds[k * cells + i]; });
        of_cells<CELLS>(8 * c, d, groups, [&](int i, int g, int at) {
            if (pl == 0 && at == 0 && i * (8 / CELLS) < n) {
                const float rest = out[g] * inv;
                const int64_t to = ((sample * s.groups + group0 + g) * a.pieces + piece) * a.blocks + block;
                a.part[to] = make_float4(m[i], rest, __builtin_fmaf(-rest * count, rest, out[groups + g]), count);
            }
        });
        __syncthreads();
    }
}

__device__ __forceinline__ double wave_sum64(double v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
// Parts of a group joined, a wavefront each: mean of the parts' means, their squared deviations around it.
__global__ __launch_bounds__(256) void k_gn_join(const float4* part, float4* stats, float* mean, float* rstd, int64_t groups, int32_t parts, float eps)
{
    const int lane = threadIdx.x & 63;
    for (int64_t g = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); g < groups; g += (int64_t)gridDim.x * 4) {
        double count = 0, sum = 0, square = 0;
        for (int i = lane; i < parts; i += 64) {
            const float4 v = part[g * parts + i];
            count += v.w;
            sum += (double)v.w * ((double)v.x + v.y);
        }
        count = wave_sum64(count);
        const double mu = wave_sum64(sum) / count;
        for (int i = lane; i < parts; i += 64) {
            const float4 v = part[g * parts + i];
            const double off = (double)v.x + v.y - mu;
            square += (double)v.z + v.w * off * off;
        }
        const double var = wave_sum64(square) / count;
        if (lane == 0) {
            const float hi = (float)mu, r = inverse_root((float)(var < 0 ? 0 : var) + eps);
            stats[g] = make_float4(hi, hi * hi > (float)var ? (float)(mu - hi) : 0.0f, r, 0.0f);
            if (mean) mean[g] = hi;
            if (rstd) rstd[g] = r;
        }
    }
}

template <typename T, bool RAGGED, bool KEPT, int CELLS> __global__ __launch_bounds__(GN_SPLIT_THREADS, 4) void k_gn_apply(GnForwardArgs<T> a)
{
    __shared__ float red[GN_SPLIT_THREADS / 64];
    const Slab& s = a.s;
    const int row_slots = KEPT ? (int)((a.k.pitch + 31) / 32 * 4) : (s.channels + 7) / 8;
    for (int64_t turn = blockIdx.x; turn < 8 * s.per_xcd; turn += gridDim.x) {
        const int64_t item = item_of(s, turn);
        if (item < 0) continue;
        int c, pl;
        place_of(s, c, pl);
        const int64_t sb = item / s.slices, sample = sb / a.blocks;
        const int slice = (int)(item - sb * s.slices), block = (int)(sb - sample * a.blocks);
        const int chunk = slice * s.slots + c, n = pl < s.lanes ? max(0, min(8, s.channels - 8 * chunk)) : 0;
        const bool live = pl < s.lanes && chunk < row_slots;
        const int p0 = block * a.rows, pixels = min(a.rows, s.pixels - p0);
        const int64_t pixel0 = sample * s.pixels + p0;
        const T* const x0 = a.x + pixel0 * a.ldx;
        const T* const x1 = n > 0 && pl < pixels ? element(x0, a.ldx, 0, pl, 8 * chunk) : x0;
        const int64_t step = (int64_t)s.lanes * a.ldx;
        Raw8<T> raw[GN_APPLY_ROWS];
#pragma unroll
        for (int u = 0; u < GN_APPLY_ROWS; ++u) {
            const bool there = n > 0 && pl + u * s.lanes < pixels;
            raw[u] = load_raw(x1 + (there ? u * step : 0), RAGGED ? (there ? n : 0) : 8);
        }
        GnChunk<T, CELLS> p;
        of_cells<CELLS>(8 * min(chunk, (s.channels - 1) / 8), s.d, s.groups, [&](int i, int g, int) {
            const float4 v = a.stats[sample * s.groups + g];
            p.mean(i, v.x, v.y);
            p.rs[i] = v.z;
        });
        load_param<T>(a.weight, a.param_f32, 8 * (int64_t)chunk, n, 1.0f, p.w);
        load_param<T>(a.bias, a.param_f32, 8 * (int64_t)chunk, n, 0.0f, p.b);
        float good = 0;
#pragma unroll
        for (int u = 0; u < GN_APPLY_ROWS; ++u) {
            const int at = pl + u * s.lanes;
            if (live && at < pixels) good += finish_chunk<T, RAGGED, KEPT, CELLS>(a, raw[u], pixel0 + at, chunk, row_slots, n, p);
            one_pixel_at_a_time();
        }
        if (a.good) {
            good = sum_block(good, red);
            if (threadIdx.x == 0) a.good[item] = good;
        }
    }
}

// goodness[sample] = sum of its parts, in their order, a wavefront each
__global__ __launch_bounds__(256) void k_gn_goodness(const float* part, float* goodness, int64_t samples, int64_t parts)
{
    const int lane = threadIdx.x & 63;
    for (int64_t b = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); b < samples; b += (int64_t)gridDim.x * 4) {
        float s = 0;
        for (int64_t i = lane; i < parts; i += 64) s += part[b * parts + i];
        s = wave_sum(s);
        if (lane == 0) goodness[b] = s;
    }
}

// ---- launches ----------------------------------------------------------------------------------------------------
size_t group_norm_workspace(int64_t samples, int64_t pixels, int64_t channels, int64_t groups)
{
    size_t most = 0;
    if (samples == 0) return FF_WS_MIN_BYTES;
    for (int size : {2, 4})
        for (bool kept : {false, true}) {
            most = std::max(most, gn_forward_floats(gn_plan(samples, pixels, channels, groups, size, kept, pitch8(channels), false), samples, groups));
            most = std::max(most, gn_backward_floats(gn_plan(samples, pixels, channels, groups, size, false, channels, true), samples, channels, groups));
        }
    return align_up(std::max<size_t>(most * sizeof(float), FF_WS_MIN_BYTES), 16);
}

template <typename T, bool RAGGED, bool KEPT, int CELLS> static hipError_t gn_forward_of(const GroupNormForwardLaunch& f, hipStream_t s)
{
    GnForwardArgs<T> a = {};
    const int64_t d = f.channels / f.groups;
    const GnPlan p = gn_plan(f.samples, f.pixels, f.channels, f.groups, sizeof(T), KEPT, pitch8(f.channels), false);
    a.x = (const T*)f.x;
    a.y = (T*)f.y;
    a.ldx = f.ldx;
    a.ldy = f.ldy;
    a.weight = f.weight;
    a.bias = f.bias;
    a.mean = f.mean;
    a.rstd = f.rstd;
    a.act = f.act;
    a.param_f32 = f.param_dtype == FF_F32;
    a.eps = f.eps;
    a.inv_m = (float)(1.0 / ((double)f.pixels * (double)d));
    if (KEPT) {
        a.k = ckpt_ptr(f.q, f.e, f.channels);
        a.r = {make_sr_key(f.seed, f.tag), f.round_mode == FF_ROUND_STOCHASTIC};
    }
    float* good;
    int64_t parts;
    if (p.whole) {
        good = (float*)f.ws;
        parts = p.cut.slices;
        a.good = f.goodness ? good : nullptr;
        a.s = slab_of(p.cut, f.samples, f.pixels, f.channels, f.groups, 1, CELLS);
        const size_t lds = gn_lds(p.cut.threads, p.cut.slots, CELLS, d);
        auto* const kernel = k_gn_forward<T, RAGGED, KEPT, CELLS>;
        GN_TRY(with_lds(kernel, lds));
        kernel<<<gn_grid(a.s), p.cut.threads, lds, s>>>(a);
        GN_TRY(hipGetLastError());
    } else {
        float4* const part = (float4*)f.ws;
        float4* const stats = part + f.samples * f.groups * p.pieces * p.blocks;
        good = (float*)(stats + f.samples * f.groups);
        parts = (int64_t)p.cut.slices * p.apply_blocks;
        a.part = part;
        a.stats = stats;
        a.pieces = p.pieces;
        a.blocks = p.blocks;
        a.rows = p.stat.lanes * GN_STAT_ROWS;
        const int cells = p.pieces > 1 || RAGGED || p.stat.slice % 8 != 0 ? 8 : gn_cells(d, false);
        a.s = slab_of(p.stat, f.samples, f.pixels, f.channels, f.groups, p.blocks, cells);
        const size_t lds = gn_lds(p.stat.threads, p.stat.slots, cells, d);
        const bool ragged = RAGGED || p.stat.slice % 8 != 0 || (p.pieces > 1 && d % 8 != 0);   // slices that end inside a chunk
        if (ragged) k_gn_stats<T, true, 8><<<gn_grid(a.s), GN_SPLIT_THREADS, lds, s>>>(a);
        else if (cells == 2) k_gn_stats<T, false, 2><<<gn_grid(a.s), GN_SPLIT_THREADS, lds, s>>>(a);
        else k_gn_stats<T, false, 8><<<gn_grid(a.s), GN_SPLIT_THREADS, lds, s>>>(a);
        GN_TRY(hipGetLastError());
        const int64_t all = f.samples * f.groups;
        k_gn_join<<<(unsigned)std::min<int64_t>((all + 3) / 4, GN_MOST_GRID), 256, 0, s>>>(part, stats, f.mean, f.rstd, all, p.pieces * p.blocks, f.eps);
        GN_TRY(hipGetLastError());
        a.good = f.goodness ? good : nullptr;
        a.blocks = p.apply_blocks;
        a.rows = p.cut.lanes * GN_APPLY_ROWS;
        a.s = slab_of(p.cut, f.samples, f.pixels, f.channels, f.groups, p.apply_blocks, CELLS);
        k_gn_apply<T, RAGGED, KEPT, CELLS><<<gn_grid(a.s), GN_SPLIT_THREADS, 0, s>>>(a);
        GN_TRY(hipGetLastError());
    }
    if (f.goodness) k_gn_goodness<<<(unsigned)std::min<int64_t>((f.samples + 3) / 4, GN_MOST_GRID), 256, 0, s>>>(good, f.goodness, f.samples, parts);
    return hipGetLastError();
}
template <typename T> static hipError_t gn_forward_typed(const GroupNormForwardLaunch& f, hipStream_t s)
{
    return by_columns(f.channels, f.groups, [&](auto ragged, auto cells) {
        return f.q ? gn_forward_of<T, decltype(ragged)::value, true, decltype(cells)::value>(f, s)
                   : gn_forward_of<T, decltype(ragged)::value, false, decltype(cells)::value>(f, s);
    });
}
hipError_t launch_group_norm_forward(const GroupNormForwardLaunch& f, hipStream_t s)
{
    return f.dtype == FF_F32    ? gn_forward_typed<float>(f, s)
           : f.dtype == FF_BF16 ? gn_forward_typed<bf16_t>(f, s)
                                : gn_forward_typed<f16_t>(f, s);
}

}  // namespace ffi
