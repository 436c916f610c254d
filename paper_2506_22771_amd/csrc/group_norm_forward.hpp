// Group norm with an activation, forward: see group_norm.hpp.
#pragma once

#include "group_norm.hpp"

namespace ffi {

// ---- forward ------------------------------------------------------------------------------------------------------------
enum GnKept { KEPT_NONE, KEPT_NEAREST, KEPT_STOCHASTIC };   // the checkpoint of h

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
    SrKey key;
    int32_t pad_steps;     // bytes of a row's exponents' pad that a chunk's lane writes, at most
    int32_t param_f32, pieces, blocks, rows;   // rows: pixels of a workgroup
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

// Where a thread's chunks go.
template <typename T, GnKept KEPT> struct GnTo {
    Walk<T> y;
    Walk<int8_t> q;
    Walk<uint8_t> e;    // the row's first byte
    uint64_t index;     // of the first pixel's chunk's first element, and how much further the next one's is
    uint64_t step;
    __device__ __forceinline__ GnTo(const GnForwardArgs<T>& a, int64_t pixel0, int pl, int chunk, bool there)
        : y(a.y, a.ldy, pixel0, a.s.lanes, there, pl, 8 * chunk), q(a.k.q, a.k.pitch, pixel0, a.s.lanes, KEPT != KEPT_NONE && there, pl, 8 * chunk),
          e(a.k.e, a.k.epitch, pixel0, a.s.lanes, KEPT != KEPT_NONE && there, pl, 0),
          index((uint64_t)(pixel0 + pl) * (uint32_t)a.s.channels + 8 * (uint32_t)chunk), step((uint64_t)a.s.lanes * (uint32_t)a.s.channels) {}
    __device__ __forceinline__ void next()
    {
        y.next();
        if constexpr (KEPT != KEPT_NONE) {
            q.next();
            e.next();
            index += step;
        }
    }
};
// A chunk: normalised, kept, activated, stored; the sum of its squares.  n of its columns exist (none: its share of the codes' pad is written).
template <typename T, bool RAGGED, GnKept KEPT, int CELLS, int ACT>
__device__ __forceinline__ float finish_chunk(const GnForwardArgs<T>& a, const GnTo<T, KEPT>& to, const Raw8<T>& raw, int chunk, int slots, int n,
                                              const GnChunk<T, CELLS>& p)
{
    float v[8], f[8];
    raw_values(raw, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p.h(v[i], i);
    if (RAGGED)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? v[i] : 0.0f;
    if constexpr (KEPT != KEPT_NONE) {
        const uint32_t top = quad_max_u32(n > 0 ? abs_max_bits(v) : 0u), e = ckpt_exponent(top);
        const u32x2 q = ckpt_codes<CELLS == 2>(v, top, e, {a.key, KEPT == KEPT_STOCHASTIC}, to.index);
        // (as ckpt_store_chunk)
        if (8 * chunk < (int)a.k.pitch) *(u32x2*)to.q.p = n > 0 ? q : u32x2{0, 0};
        uint8_t* const row = to.e.p;
        const int block = chunk >> 2;
        if ((chunk & 3) == 0 && block < a.k.blocks) row[block] = (uint8_t)e;
        int pad = a.k.blocks + chunk;
#pragma clang loop unroll(disable) vectorize(disable) interleave(disable)
        for (int i = 0; i < a.pad_steps; ++i, pad += slots)
            if (pad < (int)a.k.epitch) row[pad] = 0;
    }
    if (n <= 0) return 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_fmaf(v[i], p.w[i], p.b[i]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float d;
        act_of<T, ACT, true>(v[i], f[i], d);
        if (i & 1) one_pixel_at_a_time();
    }
    store8(to.y.p, RAGGED ? n : 8, f);
    float s = 0;
    if (a.good)   // (uniform)
#pragma unroll
        for (int i = 0; i < 8; ++i) s = !RAGGED || i < n ? __builtin_fmaf(f[i], f[i], s) : s;
    return s;
}

// U: pixels of a thread
template <typename T, bool RAGGED, GnKept KEPT, int CELLS, int ACT, int U> __global__ __launch_bounds__(1024, 4) void k_gn_forward(GnForwardArgs<T> a)
{
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const Slab& s = a.s;
    const int row_slots = KEPT != KEPT_NONE ? (int)((a.k.pitch + 31) / 32 * 4) : (s.channels + 7) / 8;
    const int item = item_of(s);
    if (item < 0) return;
    const int c = threadIdx.x % s.slots, pl = threadIdx.x / s.slots;
    const int sample = item / s.slices, slice = item - sample * s.slices, c0 = slice * s.slice;
    const int cols = min(s.slice, s.channels - c0), groups = max(1, cols / s.d);
    const int chunk = c0 / 8 + c, n = pl < s.lanes ? max(0, min(8, cols - 8 * c)) : 0;
    const bool live = pl < s.lanes && chunk < row_slots;
    const int64_t pixel0 = (int64_t)sample * s.pixels;
    // a chunk that does not exist is read from a place that does, and not used
    Walk<const T> x(a.x, a.ldx, pixel0, s.lanes, n > 0 && pl < s.pixels, pl, 8 * chunk);
    Raw8<T> raw[U];
    float v[1][CELLS] = {}, v2[2][CELLS] = {}, m[CELLS];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const bool there = n > 0 && pl + u * s.lanes < s.pixels;
        raw[u] = load_raw(x.here(there), RAGGED ? (there ? n : 0) : 8);
        x.next();
    }
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
    sum_lanes_of_groups(v, s.slots, s.lanes, s.parts, c, pl, groups, per_group, lds, out);
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
    GnChunk<T, CELLS> p;
    load_param<T>(a.weight, a.param_f32, 8 * (int64_t)chunk, n, 1.0f, p.w);
    load_param<T>(a.bias, a.param_f32, 8 * (int64_t)chunk, n, 0.0f, p.b);
    sum_lanes_of_groups(v2, s.slots, s.lanes, s.parts, c, pl, groups, per_group, lds, out);
    of_cells<CELLS>(8 * c, s.d, groups, [&](int i, int g, int at) {
        const float square = out[groups + g] * a.inv_m, rest = mean_rest(m[i], out[g] * a.inv_m, square);
        p.mean(i, m[i], rest);
        p.rs[i] = inverse_root(variance(square, rest) + a.eps);
        if (pl == 0 && at == 0 && i * (8 / CELLS) < n) {
            const int64_t to = (int64_t)sample * s.groups + (c0 / s.d + g);
            if (a.mean) a.mean[to] = m[i] + rest;
            if (a.rstd) a.rstd[to] = p.rs[i];
        }
    });
    GnTo<T, KEPT> to(a, pixel0, pl, chunk, live && pl < s.pixels);
    float good = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (live && pl + u * s.lanes < s.pixels) good += finish_chunk<T, RAGGED, KEPT, CELLS, ACT>(a, to, raw[u], chunk, row_slots, n, p);
        to.next();
        one_pixel_at_a_time();
    }
    if (a.good) {
        good = sum_block(good, lds);
        if (threadIdx.x == 0) a.good[item] = good;
    }
}

// Statistics of parts of groups: a block of pixels of a slice, which is of whole groups or a piece of one.
template <typename T, bool RAGGED, int CELLS> __global__ __launch_bounds__(GN_SPLIT_THREADS, 4) void k_gn_stats(GnForwardArgs<T> a)
{
    constexpr int U = GN_STAT_ROWS;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const Slab& s = a.s;
    const int item = item_of(s);
    if (item < 0) return;
    const int c = threadIdx.x % s.slots, pl = threadIdx.x / s.slots;
    const int sb = item / s.slices, sample = sb / a.blocks, slice = item - sb * s.slices, block = sb - sample * a.blocks;
    // the slice's columns and first group
    const bool one = a.pieces > 1;   // the slice lies in one group
    const int group0 = one ? slice / a.pieces : slice * (s.slice / s.d), piece = one ? slice - group0 * a.pieces : 0;
    const int c0 = group0 * s.d + piece * s.slice;
    const int cols = one ? min(s.slice, s.d - piece * s.slice) : min(s.slice, s.channels - c0);
    const int groups = one ? 1 : cols / s.d;
    const int n = pl < s.lanes ? max(0, min(8, cols - 8 * c)) : 0;
    const int p0 = block * a.rows, pixels = min(a.rows, s.pixels - p0);
    Walk<const T> x(a.x + c0, a.ldx, (int64_t)sample * s.pixels + p0, s.lanes, n > 0 && pl < pixels, pl, 8 * c);
    Raw8<T> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const bool there = n > 0 && pl + u * s.lanes < pixels;
        raw[u] = load_raw(x.here(there), RAGGED ? (there ? n : 0) : 8);
        x.next();
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
    sum_lanes_of_groups(v, s.slots, s.lanes, s.parts, c, pl, groups, per_group, lds, out);
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
    sum_lanes_of_groups(v2, s.slots, s.lanes, s.parts, c, pl, groups, per_group, lds, out);
    of_cells<CELLS>(8 * c, d, groups, [&](int i, int g, int at) {
        if (pl == 0 && at == 0 && i * (8 / CELLS) < n) {
            const float rest = out[g] * inv;
            const int64_t to = (((int64_t)sample * s.groups + group0 + g) * a.pieces + piece) * a.blocks + block;
            a.part[to] = make_float4(m[i], rest, __builtin_fmaf(-rest * count, rest, out[groups + g]), count);
        }
    });
}

template <typename T, bool RAGGED, GnKept KEPT, int CELLS, int ACT> __global__ __launch_bounds__(GN_SPLIT_THREADS, 4) void k_gn_apply(GnForwardArgs<T> a)
{
    __shared__ float red[GN_SPLIT_THREADS / 64];
    const Slab& s = a.s;
    const int row_slots = KEPT != KEPT_NONE ? (int)((a.k.pitch + 31) / 32 * 4) : (s.channels + 7) / 8;
    const int item = item_of(s);
    if (item < 0) return;
    const int c = threadIdx.x % s.slots, pl = threadIdx.x / s.slots;
    const int sb = item / s.slices, sample = sb / a.blocks, slice = item - sb * s.slices, block = sb - sample * a.blocks;
    const int chunk = slice * s.slots + c, n = pl < s.lanes ? max(0, min(8, s.channels - 8 * chunk)) : 0;
    const bool live = pl < s.lanes && chunk < row_slots;
    const int p0 = block * a.rows, pixels = min(a.rows, s.pixels - p0);
    const int64_t pixel0 = (int64_t)sample * s.pixels + p0;
    Walk<const T> x(a.x, a.ldx, pixel0, s.lanes, n > 0 && pl < pixels, pl, 8 * chunk);
    Raw8<T> raw[GN_APPLY_ROWS];
#pragma unroll
    for (int u = 0; u < GN_APPLY_ROWS; ++u) {
        const bool there = n > 0 && pl + u * s.lanes < pixels;
        raw[u] = load_raw(x.here(there), RAGGED ? (there ? n : 0) : 8);
        x.next();
    }
    GnChunk<T, CELLS> p;
    of_cells<CELLS>(8 * min(chunk, (s.channels - 1) / 8), s.d, s.groups, [&](int i, int g, int) {
        const float4 v = a.stats[(int64_t)sample * s.groups + g];
        p.mean(i, v.x, v.y);
        p.rs[i] = v.z;
    });
    load_param<T>(a.weight, a.param_f32, 8 * (int64_t)chunk, n, 1.0f, p.w);
    load_param<T>(a.bias, a.param_f32, 8 * (int64_t)chunk, n, 0.0f, p.b);
    GnTo<T, KEPT> to(a, pixel0, pl, chunk, live && pl < pixels);
    float good = 0;
#pragma unroll
    for (int u = 0; u < GN_APPLY_ROWS; ++u) {
        if (live && pl + u * s.lanes < pixels) good += finish_chunk<T, RAGGED, KEPT, CELLS, ACT>(a, to, raw[u], chunk, row_slots, n, p);
        to.next();
        one_pixel_at_a_time();
    }
    if (a.good) {
        good = sum_block(good, red);
        if (threadIdx.x == 0) a.good[item] = good;
    }
}

// ---- launches ----------------------------------------------------------------------------------------------------
template <typename T, bool RAGGED, GnKept KEPT, int CELLS, int ACT> static hipError_t gn_forward_of(const GroupNormForwardLaunch& f, hipStream_t s)
{
    GnForwardArgs<T> a = {};
    const int64_t d = f.channels / f.groups;
    const GnPlan p = gn_plan(f.samples, f.pixels, f.channels, f.groups, sizeof(T), KEPT != KEPT_NONE, pitch8(f.channels), false);
    a.x = (const T*)f.x;
    a.y = (T*)f.y;
    a.ldx = f.ldx;
    a.ldy = f.ldy;
    a.weight = f.weight;
    a.bias = f.bias;
    a.mean = f.mean;
    a.rstd = f.rstd;
    a.param_f32 = f.param_dtype == FF_F32;
    a.eps = f.eps;
    a.inv_m = (float)(1.0 / ((double)f.pixels * (double)d));
    if (KEPT != KEPT_NONE) {
        a.k = ckpt_ptr(f.q, f.e, f.channels);
        a.key = make_sr_key(f.seed, f.tag);
        const int64_t row_slots = (a.k.pitch + 31) / 32 * 4;
        a.pad_steps = (int32_t)((a.k.epitch - a.k.blocks + row_slots - 1) / row_slots);
    }
    float* good;
    int64_t parts;
    if (p.whole) {
        parts = p.cut.slices;
        good = parts == 1 ? f.goodness : (float*)f.ws;   // (one part is the sum)
        a.good = f.goodness ? good : nullptr;
        a.s = slab_of(p.cut, f.samples, f.pixels, f.channels, f.groups, 1, CELLS);
        const size_t lds = gn_lds(p.cut.threads, p.cut.slots, CELLS, d);
        // slabs of a quarter of the pixels by a kernel of no more (45 x 33x33 x 1 bf16 forward 14.0 us, by the other 18.7; 138 x 5x5 x 23 backward 10.0 and 12.1)
        constexpr int U = gn_rows(sizeof(T), false), FEW = U / 4;
        auto* const kernel = p.cut.lanes * FEW >= f.pixels ? k_gn_forward<T, RAGGED, KEPT, CELLS, ACT, FEW> : k_gn_forward<T, RAGGED, KEPT, CELLS, ACT, U>;
        GN_TRY(with_lds(kernel, lds));
        GN_TRY(launch_items(a, [&](unsigned grid, const auto& part) { kernel<<<grid, p.cut.threads, lds, s>>>(part); }));
    } else {
        float4* const part = (float4*)f.ws;
        float4* const stats = part + f.samples * f.groups * p.pieces * p.blocks;
        parts = (int64_t)p.cut.slices * p.apply_blocks;
        good = parts == 1 ? f.goodness : (float*)(stats + f.samples * f.groups);
        a.part = part;
        a.stats = stats;
        a.pieces = p.pieces;
        a.blocks = p.blocks;
        a.rows = p.stat.lanes * GN_STAT_ROWS;
        const int cells = p.pieces > 1 || p.stat.slice % 8 != 0 ? 8 : gn_cells(f.channels, d, false);
        a.s = slab_of(p.stat, f.samples, f.pixels, f.channels, f.groups, p.blocks, cells);
        const size_t lds = gn_lds(p.stat.threads, p.stat.slots, cells, d);
        const bool ragged = RAGGED || p.stat.slice % 8 != 0 || (p.pieces > 1 && d % 8 != 0);   // slices that end inside a chunk
        GN_TRY(launch_items(a, [&](unsigned grid, const auto& part) {
            if (ragged) k_gn_stats<T, true, 8><<<grid, GN_SPLIT_THREADS, lds, s>>>(part);
            else if (cells == 2) k_gn_stats<T, false, 2><<<grid, GN_SPLIT_THREADS, lds, s>>>(part);
            else k_gn_stats<T, false, 8><<<grid, GN_SPLIT_THREADS, lds, s>>>(part);
        }));
        GN_TRY(launch_gn_join(part, stats, f, p.pieces * p.blocks, s));
        a.good = f.goodness ? good : nullptr;
        a.blocks = p.apply_blocks;
        a.rows = p.cut.lanes * GN_APPLY_ROWS;
        a.s = slab_of(p.cut, f.samples, f.pixels, f.channels, f.groups, p.apply_blocks, CELLS);
        GN_TRY(launch_items(a, [&](unsigned grid, const auto& part) { k_gn_apply<T, RAGGED, KEPT, CELLS, ACT><<<grid, GN_SPLIT_THREADS, 0, s>>>(part); }));
    }
    return f.goodness && parts > 1 ? launch_gn_goodness(good, f.goodness, f.samples, parts, s) : hipSuccess;
}
template <typename T> hipError_t gn_forward_typed(const GroupNormForwardLaunch& f, hipStream_t s)
{
    return by_columns(f.channels, f.groups, [&](auto ragged, auto cells) {
        return by_activation(f.act, [&](auto act) {
            constexpr bool RAGGED = decltype(ragged)::value;
            constexpr int CELLS = decltype(cells)::value, ACT = decltype(act)::value;
            return !f.q                                      ? gn_forward_of<T, RAGGED, KEPT_NONE, CELLS, ACT>(f, s)
                   : f.round_mode == FF_ROUND_STOCHASTIC ? gn_forward_of<T, RAGGED, KEPT_STOCHASTIC, CELLS, ACT>(f, s)
                                                         : gn_forward_of<T, RAGGED, KEPT_NEAREST, CELLS, ACT>(f, s);
        });
    });
}

}  // namespace ffi
