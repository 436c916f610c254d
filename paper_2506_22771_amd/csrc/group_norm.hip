// Group norm with an activation over channels-last maps, forward and backward.
//
//   per sample and group, over its d channels at all P pixels:  mean, rstd = 1 / sqrt(1/(P d) sum (x - mean)^2 + eps),  h = (x - mean) rstd
//   z = h gamma + beta,  y = f(z),  G = sum over the sample of f(z)^2
//   dz = (dy + 2 c f(z)) f'(z),  dgamma = sum over pixels and samples of dz h,  dbeta = sum of dz
//   dx = rstd (g - 1/(P d) sum over the group of g - h 1/(P d) sum over the group of g h),  g = gamma dz
//
// Statistics, products and sums are fp32 (the means of parts of a group are joined in 64 bits); y and dx are rounded once.  As in the layer norm, the mean of
// the deviations is taken out of groups farther from zero than they are wide (norm_math.hpp).
//
// Memory bounds all of it.  A workgroup's threads lie over a slab of whole groups: a chunk of eight columns is a thread's own from pixel to pixel, so that
// parameters and sums of columns stay in registers, and sums meet in LDS once.  Where such a slab fits the registers of a workgroup, everything is read once
// (one launch, `whole` below; group_norm_plan.hpp).  Else a first launch sums parts of groups, a small one joins them, and a third reads again and applies.
// The sums of all samples, dgamma and dbeta, are a launch of their own over sums of columns per sample.
#include "act.hpp"
#include "blocks.hpp"
#include "group_norm_plan.hpp"
#include "norm_math.hpp"

namespace ffi {

// ---- slabs ------------------------------------------------------------------------------------------------------------
struct Slab {
    int32_t slots, lanes, slice, slices;   // see GnCut
    int32_t pixels, channels, groups, d;
    int32_t cells_per_chunk;   // sums of a chunk that are kept apart: 1 where it lies in one group, 2 where its halves do, else 8
    int32_t parts;             // threads that share the sum of a cell over the lanes, at most
    int64_t items, per_xcd;    // workgroups' work: (sample, [block of pixels,] slice)
};
// Items in turn to the eight XCDs, so that neighbours, which share cache lines, meet in one L2; -1: none.
__device__ __forceinline__ int64_t item_of(const Slab& s, int64_t turn)
{
    const int64_t i = (turn & 7) * s.per_xcd + (turn >> 3);
    return i < s.items ? i : -1;
}

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Sums over the lanes of K values of each of a chunk's columns: `cell(k, i)` below are the sums of cell i (a column, or the columns of a chunk or half of one
// that lie in one group).  lds: K cells (lanes + parts + 1) floats.  A barrier ends it.
template <int K, int THREADS> struct CellSums {
    float* lds;
    int cells;
    __device__ __forceinline__ float cell(int k, int i) const { return lds[k * cells + i]; }
};
template <int K, int THREADS>
__device__ __forceinline__ CellSums<K, THREADS> sum_cells(float (&v)[K][8], int per, int slots, int lanes, int most_parts, int c, int pl, float* lds)
{
    const int cells = slots * per, parts = max(1, min(most_parts, THREADS / (K * cells)));
    float* const all = lds + K * cells * (1 + most_parts);
    if (pl < lanes) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float* const to = all + (k * lanes + pl) * cells + c * per;
            if (per == 1) {
                *to = ((v[k][0] + v[k][1]) + (v[k][2] + v[k][3])) + ((v[k][4] + v[k][5]) + (v[k][6] + v[k][7]));
            } else if (per == 2) {
                to[0] = (v[k][0] + v[k][1]) + (v[k][2] + v[k][3]);
                to[1] = (v[k][4] + v[k][5]) + (v[k][6] + v[k][7]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) to[i] = v[k][i];
            }
        }
    }
    __syncthreads();
    float* const some = lds + K * cells;
    for (int t = threadIdx.x; t < K * cells * parts; t += THREADS) {
        const int part = t / (K * cells), kc = t - part * (K * cells), k = kc / cells, i = kc - k * cells;
        float s = 0;
        for (int l = part; l < lanes; l += parts) s += all[(k * lanes + l) * cells + i];
        some[t] = s;
    }
    __syncthreads();
    for (int t = threadIdx.x; t < K * cells; t += THREADS) {
        float s = 0;
        for (int part = 0; part < parts; ++part) s += some[part * (K * cells) + t];
        lds[t] = s;
    }
    __syncthreads();
    return {lds, cells};
}
// Sums over the `n` cells of each of `groups` groups, by value(k, cell), into out[k * groups + g].  A barrier ends it.
template <int K, int THREADS, typename F> __device__ __forceinline__ void sum_groups(int groups, int n, float* out, F&& value)
{
    if (n <= 16) {
        for (int t = threadIdx.x; t < K * groups; t += THREADS) {
            const int k = t / groups, g = t - k * groups;
            float s = 0;
            for (int i = 0; i < n; ++i) s += value(k, g * n + i);
            out[t] = s;
        }
    } else {
        for (int t = threadIdx.x >> 6; t < K * groups; t += THREADS / 64) {
            const int k = t / groups, g = t - k * groups;
            float s = 0;
            for (int i = threadIdx.x & 63; i < n; i += 64) s += value(k, g * n + i);
            s = wave_sum(s);
            if ((threadIdx.x & 63) == 0) out[t] = s;
        }
    }
    __syncthreads();
}

// Sum of a workgroup's values, in thread 0.  red: a word per wavefront.  A barrier begins it.
template <int THREADS> __device__ __forceinline__ float sum_block(float v, float* red)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0;
    if (threadIdx.x == 0)
        for (int w = 0; w < THREADS / 64; ++w) s += red[w];
    return s;
}

// What each of a chunk's columns takes of its group: value(group) for groups counted from the slice's first column on.
template <typename F> __device__ __forceinline__ void of_columns(int first, int d, int groups, F&& each)
{
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

template <typename T> __device__ __forceinline__ void activate(int act, const float z[8], float f[8])
{
    float d;
    switch (act) {   // (uniform)
        case FF_ACT_RELU:
#pragma unroll
            for (int i = 0; i < 8; ++i) act_of<T, FF_ACT_RELU, true>(z[i], f[i], d);
            break;
        case FF_ACT_GELU:
#pragma unroll
            for (int i = 0; i < 8; ++i) act_of<T, FF_ACT_GELU, true>(z[i], f[i], d);
            break;
        case FF_ACT_SILU:
#pragma unroll
            for (int i = 0; i < 8; ++i) act_of<T, FF_ACT_SILU, true>(z[i], f[i], d);
            break;
        default:
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = z[i];
    }
}

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

// One chunk: normalised, kept, activated, stored; the sum of its squares.  n of its columns exist (none: its share of the codes' pad is written).
template <typename T, bool RAGGED, bool KEPT>
__device__ __forceinline__ float finish_chunk(const GnForwardArgs<T>& a, const Raw8<T>& raw, int64_t pixel, int chunk, int slots, int n, const float m[8],
                                              const float rest[8], const float rs[8], const float w[8], const float b[8])
{
    float v[8], f[8];
    raw_values(raw, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (v[i] - m[i] - rest[i]) * rs[i];
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
    for (int i = 0; i < 8; ++i) v[i] = __builtin_fmaf(v[i], w[i], b[i]);
    activate<T>(a.act, v, f);
    store8(a.y + (pixel * a.ldy + 8 * chunk), RAGGED ? n : 8, f);
    if (!a.good) return 0.0f;
    float s = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (!RAGGED || i < n) s = __builtin_fmaf(f[i], f[i], s);
    return s;
}

template <typename T, bool RAGGED, bool KEPT, int THREADS, int U> __global__ __launch_bounds__(THREADS) void k_gn_forward(GnForwardArgs<T> a)
{
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const Slab& s = a.s;
    const int c = threadIdx.x % s.slots, pl = threadIdx.x / s.slots;
    const int row_slots = KEPT ? (int)((a.k.pitch + 31) / 32 * 4) : (s.channels + 7) / 8;
    for (int64_t turn = blockIdx.x; turn < 8 * s.per_xcd; turn += gridDim.x) {
        const int64_t item = item_of(s, turn);
        if (item < 0) continue;
        const int64_t sample = item / s.slices;
        const int slice = (int)(item - sample * s.slices), c0 = slice * s.slice;
        const int cols = min(s.slice, s.channels - c0), groups = max(1, cols / s.d);
        const int chunk = c0 / 8 + c, n = pl < s.lanes ? max(0, min(8, cols - 8 * c)) : 0;
        const bool live = pl < s.lanes && chunk < row_slots;
        const int64_t pixel0 = sample * s.pixels;
        const T* const x = a.x + pixel0 * a.ldx;
        Raw8<T> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = pl + u * s.lanes;
            const bool there = n > 0 && p < s.pixels;
            if (RAGGED) raw[u] = load_raw(element(x, a.ldx, 0, there ? p : 0, there ? 8 * chunk : 0), there ? n : 0);
            else raw[u] = load_raw(element(x, a.ldx, 0, there ? p : 0, there ? 8 * chunk : 0), 8);
        }
        float v[1][8] = {}, m[8], rest[8], rs[8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (n > 0 && pl + u * s.lanes < s.pixels) {
                float t[8];
                raw_values(raw[u], t);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[0][i] += t[i];
            }
            opaque(raw[u]);
        }
        const int per_group = s.d * s.cells_per_chunk / 8;
        float* const out = lds + 2 * s.slots * s.cells_per_chunk * (1 + s.parts + s.lanes);
        {
            const auto sums = sum_cells<1, THREADS>(v, s.cells_per_chunk, s.slots, s.lanes, s.parts, c, pl, lds);
            sum_groups<1, THREADS>(groups, per_group, out, [&](int k, int i) { return sums.cell(k, i); });
        }
        of_columns(8 * c, s.d, groups, [&](int i, int g, int) { m[i] = out[g] * a.inv_m; });
        float v2[2][8] = {};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (n > 0 && pl + u * s.lanes < s.pixels) {
                float t[8];
                raw_values(raw[u], t);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float dev = !RAGGED || i < n ? t[i] - m[i] : 0.0f;
                    v2[0][i] += dev;
                    v2[1][i] = __builtin_fmaf(dev, dev, v2[1][i]);
                }
            }
            opaque(raw[u]);
        }
        {
            const auto sums = sum_cells<2, THREADS>(v2, s.cells_per_chunk, s.slots, s.lanes, s.parts, c, pl, lds);
            sum_groups<2, THREADS>(groups, per_group, out, [&](int k, int i) { return sums.cell(k, i); });
        }
        of_columns(8 * c, s.d, groups, [&](int i, int g, int at) {
            const float square = out[groups + g] * a.inv_m;
            rest[i] = mean_rest(m[i], out[g] * a.inv_m, square);
            rs[i] = inverse_root(variance(square, rest[i]) + a.eps);
            if (pl == 0 && at == 0 && i < n) {
                const int64_t to = sample * s.groups + (c0 / s.d + g);
                if (a.mean) a.mean[to] = m[i] + rest[i];
                if (a.rstd) a.rstd[to] = rs[i];
            }
        });
        float w[8], b[8], good = 0;
        load_param<T>(a.weight, a.param_f32, 8 * (int64_t)chunk, n, 1.0f, w);
        load_param<T>(a.bias, a.param_f32, 8 * (int64_t)chunk, n, 0.0f, b);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = pl + u * s.lanes;
            if (live && p < s.pixels) good += finish_chunk<T, RAGGED, KEPT>(a, raw[u], pixel0 + p, chunk, row_slots, n, m, rest, rs, w, b);
        }
        if (a.good) {
            good = sum_block<THREADS>(good, lds);
            if (threadIdx.x == 0) a.good[item] = good;
        }
        __syncthreads();   // (the next item's sums go where this one's lie)
    }
}

// Statistics of parts of groups: a block of pixels of a slice, which is of whole groups or a piece of one.
template <typename T, int U> __global__ __launch_bounds__(GN_SPLIT_THREADS) void k_gn_stats(GnForwardArgs<T> a)
{
    constexpr int THREADS = GN_SPLIT_THREADS;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const Slab& s = a.s;
    const int c = threadIdx.x % s.slots, pl = threadIdx.x / s.slots;
    for (int64_t turn = blockIdx.x; turn < 8 * s.per_xcd; turn += gridDim.x) {
        const int64_t item = item_of(s, turn);
        if (item < 0) continue;
        const int64_t sb = item / s.slices, sample = sb / a.blocks;
        const int slice = (int)(item - sb * s.slices), block = (int)(sb - sample * a.blocks);
        // the slice's columns and first group
        const int group0 = a.pieces == 1 ? slice * (s.slice / s.d) : slice / a.pieces, piece = a.pieces == 1 ? 0 : slice - group0 * a.pieces;
        const int c0 = group0 * s.d + piece * s.slice;
        const int cols = a.pieces == 1 ? min(s.slice, s.channels - c0) : min(s.slice, s.d - piece * s.slice);
        const int groups = a.pieces == 1 ? cols / s.d : 1;
        const int n = pl < s.lanes ? max(0, min(8, cols - 8 * c)) : 0;
        const int p0 = block * a.rows, pixels = min(a.rows, s.pixels - p0);
        const T* const x = a.x + (sample * s.pixels + p0) * a.ldx + c0;
        Raw8<T> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = pl + u * s.lanes;
            const bool there = n > 0 && p < pixels;
            raw[u] = load_raw(element(x, a.ldx, 0, there ? p : 0, there ? 8 * c : 0), there ? n : 0);
        }
        float v[1][8] = {}, m[8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float t[8];
            raw_values(raw[u], t);   // (zeros where there is none)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[0][i] += t[i];
            opaque(raw[u]);
        }
        const int per_group = a.pieces == 1 ? s.d * s.cells_per_chunk / 8 : s.slots * s.cells_per_chunk;
        const int d = a.pieces == 1 ? s.d : 8 * s.slots;
        const float count = (float)(pixels * (a.pieces == 1 ? s.d : cols)), inv = 1.0f / count;
        float* const out = lds + 2 * s.slots * s.cells_per_chunk * (1 + s.parts + s.lanes);
        {
            const auto sums = sum_cells<1, THREADS>(v, s.cells_per_chunk, s.slots, s.lanes, s.parts, c, pl, lds);
            sum_groups<1, THREADS>(groups, per_group, out, [&](int k, int i) { return sums.cell(k, i); });
        }
        of_columns(8 * c, d, groups, [&](int i, int g, int) { m[i] = out[g] * inv; });
        float v2[2][8] = {};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (pl + u * s.lanes < pixels) {
                float t[8];
                raw_values(raw[u], t);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float dev = i < n ? t[i] - m[i] : 0.0f;
                    v2[0][i] += dev;
                    v2[1][i] = __builtin_fmaf(dev, dev, v2[1][i]);
                }
            }
        }
        {
            const auto sums = sum_cells<2, THREADS>(v2, s.cells_per_chunk, s.slots, s.lanes, s.parts, c, pl, lds);
            sum_groups<2, THREADS>(groups, per_group, out, [&](int k, int i) { return sums.cell(k, i); });
        }
        of_columns(8 * c, d, groups, [&](int i, int g, int at) {
            if (pl == 0 && at == 0 && i < n) {
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

template <typename T, bool RAGGED, bool KEPT> __global__ __launch_bounds__(GN_SPLIT_THREADS) void k_gn_apply(GnForwardArgs<T> a)
{
    __shared__ float red[GN_SPLIT_THREADS / 64];
    const Slab& s = a.s;
    const int c = threadIdx.x % s.slots, pl = threadIdx.x / s.slots;
    const int row_slots = KEPT ? (int)((a.k.pitch + 31) / 32 * 4) : (s.channels + 7) / 8;
    for (int64_t turn = blockIdx.x; turn < 8 * s.per_xcd; turn += gridDim.x) {
        const int64_t item = item_of(s, turn);
        if (item < 0) continue;
        const int64_t sb = item / s.slices, sample = sb / a.blocks;
        const int slice = (int)(item - sb * s.slices), block = (int)(sb - sample * a.blocks);
        const int chunk = slice * s.slots + c, n = pl < s.lanes ? max(0, min(8, s.channels - 8 * chunk)) : 0;
        const bool live = pl < s.lanes && chunk < row_slots;
        const int p0 = block * a.rows, pixels = min(a.rows, s.pixels - p0);
        const int64_t pixel0 = sample * s.pixels + p0;
        const T* const x = a.x + pixel0 * a.ldx;
        Raw8<T> raw[GN_APPLY_ROWS];
#pragma unroll
        for (int u = 0; u < GN_APPLY_ROWS; ++u) {
            const int p = pl + u * s.lanes;
            const bool there = n > 0 && p < pixels;
            if (RAGGED) raw[u] = load_raw(element(x, a.ldx, 0, there ? p : 0, there ? 8 * chunk : 0), there ? n : 0);
            else raw[u] = load_raw(element(x, a.ldx, 0, there ? p : 0, there ? 8 * chunk : 0), 8);
        }
        float m[8], rest[8], rs[8], w[8], b[8], good = 0;
        of_columns(8 * min(chunk, (s.channels - 1) / 8), s.d, s.groups, [&](int i, int g, int) {
            const float4 v = a.stats[sample * s.groups + g];
            m[i] = v.x;
            rest[i] = v.y;
            rs[i] = v.z;
        });
        load_param<T>(a.weight, a.param_f32, 8 * (int64_t)chunk, n, 1.0f, w);
        load_param<T>(a.bias, a.param_f32, 8 * (int64_t)chunk, n, 0.0f, b);
#pragma unroll
        for (int u = 0; u < GN_APPLY_ROWS; ++u) {
            const int p = pl + u * s.lanes;
            if (live && p < pixels) good += finish_chunk<T, RAGGED, KEPT>(a, raw[u], pixel0 + p, chunk, row_slots, n, m, rest, rs, w, b);
        }
        if (a.good) {
            good = sum_block<GN_SPLIT_THREADS>(good, red);
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
    int32_t act, param_f32, blocks, rows;
    float inv_m;
};

// What a thread holds of one pixel.
template <typename T, bool FROM_X> struct GnPixel {
    Raw8<T> dy, x;
    u32x2 q;
    uint32_t e;
};
template <typename T, bool RAGGED, bool FROM_X>
__device__ __forceinline__ void load_pixel(const GnBackwardArgs<T>& a, GnPixel<T, FROM_X>& v, int64_t pixel, int chunk, int n)
{
    // n == 0: what is read is not used, and lies in the first chunk of the pixel's row
    const int at = n > 0 ? chunk : 0, m = RAGGED ? n : 8;
    raw_zero(v.dy);
    if (a.dy) v.dy = load_raw(a.dy + (pixel * a.lddy + 8 * at), m);
    if constexpr (FROM_X) {
        v.x = load_raw(a.x + (pixel * a.ldx + 8 * at), m);
    } else {
        v.q = *(const u32x2*)(a.k.q + (pixel * a.k.pitch + 8 * at));
        v.e = a.k.e[pixel * a.k.epitch + (at >> 2)];
    }
}
// h and dz of one pixel
template <typename T, bool FROM_X>
__device__ __forceinline__ void dz_of(const GnBackwardArgs<T>& a, const GnPixel<T, FROM_X>& v, float c2, const float m[8], const float rs[8], const float w[8],
                                      const float b[8], float h[8], float dz[8])
{
    if constexpr (FROM_X) {
        raw_values(v.x, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = (h[i] - m[i]) * rs[i];
    } else {
        ckpt_values(v.q, v.e, h);
    }
    raw_values(v.dy, dz);
    auto through = [&](auto kind) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float f, d;
            act_of<T, decltype(kind)::value, true>(__builtin_fmaf(h[i], w[i], b[i]), f, d);
            dz[i] = __builtin_fmaf(c2, f, dz[i]) * d;
        }
    };
    switch (a.act) {   // (uniform)
        case FF_ACT_RELU: through(std::integral_constant<int, FF_ACT_RELU>()); break;
        case FF_ACT_GELU: through(std::integral_constant<int, FF_ACT_GELU>()); break;
        case FF_ACT_SILU: through(std::integral_constant<int, FF_ACT_SILU>()); break;
        default:
            if (a.coeff) through(std::integral_constant<int, FF_ACT_IDENTITY>());
    }
}
template <typename T, bool RAGGED>
__device__ __forceinline__ void store_dx(const GnBackwardArgs<T>& a, int64_t pixel, int chunk, int n, const float h[8], const float dz[8], const float rs[8],
                                         const float w[8], const float sg[8], const float sh[8])
{
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = rs[i] * (__builtin_fmaf(-h[i], sh[i], w[i] * dz[i] - sg[i]));
    store8(a.dx + (pixel * a.lddx + 8 * chunk), RAGGED ? n : 8, v);
}

template <typename T, bool RAGGED, bool FROM_X, int THREADS, int U> __global__ __launch_bounds__(THREADS) void k_gn_backward(GnBackwardArgs<T> a)
{
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const Slab& s = a.s;
    const int c = threadIdx.x % s.slots, pl = threadIdx.x / s.slots;
    for (int64_t turn = blockIdx.x; turn < 8 * s.per_xcd; turn += gridDim.x) {
        const int64_t item = item_of(s, turn);
        if (item < 0) continue;
        const int64_t sample = item / s.slices;
        const int slice = (int)(item - sample * s.slices), c0 = slice * s.slice;
        const int cols = min(s.slice, s.channels - c0), groups = max(1, cols / s.d);
        const int chunk = c0 / 8 + c, n = pl < s.lanes ? max(0, min(8, cols - 8 * c)) : 0;
        const int64_t pixel0 = sample * s.pixels;
        GnPixel<T, FROM_X> px[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = pl + u * s.lanes;
            const bool there = n > 0 && p < s.pixels;
            load_pixel<T, RAGGED, FROM_X>(a, px[u], pixel0 + (there ? p : 0), chunk, there ? n : 0);
        }
        float w[8], b[8], m[8], rs[8], v[2][8] = {};
        load_param<T>(a.weight, a.param_f32, 8 * (int64_t)chunk, n, 1.0f, w);
        load_param<T>(a.bias, a.param_f32, 8 * (int64_t)chunk, n, 0.0f, b);
        of_columns(8 * c, s.d, groups, [&](int i, int g, int) {
            const int64_t from = sample * s.groups + (c0 / s.d + g);
            m[i] = FROM_X ? a.mean[from] : 0.0f;
            rs[i] = a.rstd[from];
        });
        const float c2 = a.coeff ? 2.0f * a.coeff[sample] : 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (n > 0 && pl + u * s.lanes < s.pixels) {
                float h[8], dz[8];
                dz_of(a, px[u], c2, m, rs, w, b, h, dz);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[0][i] += !RAGGED || i < n ? dz[i] : 0.0f;
                    v[1][i] = __builtin_fmaf(!RAGGED || i < n ? dz[i] : 0.0f, !RAGGED || i < n ? h[i] : 0.0f, v[1][i]);
                }
            }
            opaque(px[u].dy);
            if constexpr (FROM_X) opaque(px[u].x);
            else opaque(px[u].q);
        }
        float* const out = lds + 2 * s.slots * 8 * (1 + s.parts + s.lanes);
        float* const ws = out + 2 * ((s.slots * 8 + s.d - 1) / s.d + 1);
        if (pl == 0)
#pragma unroll
            for (int i = 0; i < 8; ++i) ws[8 * c + i] = w[i];
        const auto sums = sum_cells<2, THREADS>(v, 8, s.slots, s.lanes, s.parts, c, pl, lds);
        if (a.sums)
            for (int t = threadIdx.x; t < cols; t += THREADS) a.sums[sample * s.channels + c0 + t] = make_float2(sums.cell(0, t), sums.cell(1, t));
        if (a.dx) {
            sum_groups<2, THREADS>(groups, s.d, out, [&](int k, int i) { return ws[i] * sums.cell(k, i); });
            float sg[8], sh[8];
            of_columns(8 * c, s.d, groups, [&](int i, int g, int) {
                sg[i] = out[g] * a.inv_m;
                sh[i] = out[groups + g] * a.inv_m;
            });
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int p = pl + u * s.lanes;
                if (n > 0 && p < s.pixels) {
                    float h[8], dz[8];
                    dz_of(a, px[u], c2, m, rs, w, b, h, dz);
                    store_dx<T, RAGGED>(a, pixel0 + p, chunk, n, h, dz, rs, w, sg, sh);
                }
            }
        }
        __syncthreads();
    }
}

// Sums of columns over a block of pixels.
template <typename T, bool RAGGED, bool FROM_X> __global__ __launch_bounds__(GN_SPLIT_THREADS) void k_gn_backward_sums(GnBackwardArgs<T> a)
{
    constexpr int THREADS = GN_SPLIT_THREADS, U = 2;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const Slab& s = a.s;
    const int c = threadIdx.x % s.slots, pl = threadIdx.x / s.slots;
    for (int64_t turn = blockIdx.x; turn < 8 * s.per_xcd; turn += gridDim.x) {
        const int64_t item = item_of(s, turn);
        if (item < 0) continue;
        const int64_t sb = item / s.slices, sample = sb / a.blocks;
        const int slice = (int)(item - sb * s.slices), block = (int)(sb - sample * a.blocks);
        const int chunk = slice * s.slots + c, c0 = slice * s.slice, cols = min(s.slice, s.channels - c0);
        const int n = pl < s.lanes ? max(0, min(8, s.channels - 8 * chunk)) : 0;
        const int p0 = block * a.rows, pixels = min(a.rows, s.pixels - p0);
        const int64_t pixel0 = sample * s.pixels + p0;
        float w[8], b[8], m[8], rs[8], v[2][8] = {};
        load_param<T>(a.weight, a.param_f32, 8 * (int64_t)chunk, n, 1.0f, w);
        load_param<T>(a.bias, a.param_f32, 8 * (int64_t)chunk, n, 0.0f, b);
        of_columns(8 * min(chunk, (s.channels - 1) / 8), s.d, s.groups, [&](int i, int g, int) {
            m[i] = FROM_X ? a.mean[sample * s.groups + g] : 0.0f;
            rs[i] = a.rstd[sample * s.groups + g];
        });
        const float c2 = a.coeff ? 2.0f * a.coeff[sample] : 0.0f;
        for (int p1 = pl; p1 - pl < pixels; p1 += U * s.lanes) {
            GnPixel<T, FROM_X> px[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int p = p1 + u * s.lanes;
                const bool there = n > 0 && p < pixels;
                load_pixel<T, RAGGED, FROM_X>(a, px[u], pixel0 + (there ? p : 0), chunk, there ? n : 0);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (n > 0 && p1 + u * s.lanes < pixels) {
                    float h[8], dz[8];
                    dz_of(a, px[u], c2, m, rs, w, b, h, dz);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        v[0][i] += !RAGGED || i < n ? dz[i] : 0.0f;
                        v[1][i] = __builtin_fmaf(!RAGGED || i < n ? dz[i] : 0.0f, !RAGGED || i < n ? h[i] : 0.0f, v[1][i]);
                    }
                }
            }
        }
        const auto sums = sum_cells<2, THREADS>(v, 8, s.slots, s.lanes, s.parts, c, pl, lds);
        for (int t = threadIdx.x; t < cols; t += THREADS) a.sums[sb * s.channels + c0 + t] = make_float2(sums.cell(0, t), sums.cell(1, t));
        __syncthreads();
    }
}

// Sums of a sample's blocks, a wavefront for a group: sums of its columns, and those of the group by its size.
template <typename T>
__global__ __launch_bounds__(256) void k_gn_backward_join(const float2* part, float2* sums, float2* group, const void* weight, int param_f32, int64_t samples,
                                                          int32_t groups, int32_t d, int32_t blocks, float inv_m)
{
    const int lane = threadIdx.x & 63, channels = groups * d;
    for (int64_t sg = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); sg < samples * groups; sg += (int64_t)gridDim.x * 4) {
        const int64_t sample = sg / groups;
        const int c0 = (int)(sg - sample * groups) * d;
        float2 of_group = make_float2(0, 0);
        for (int i = lane; i < d; i += 64) {
            float2 t = make_float2(0, 0);
#pragma unroll 8
            for (int b = 0; b < blocks; ++b) {
                const float2 v = part[(sample * blocks + b) * channels + c0 + i];
                t.x += v.x;
                t.y += v.y;
            }
            float w[8];
            load_param<T>(weight, param_f32, c0 + i, 1, 1.0f, w);
            sums[sample * channels + c0 + i] = t;
            of_group.x = __builtin_fmaf(w[0], t.x, of_group.x);
            of_group.y = __builtin_fmaf(w[0], t.y, of_group.y);
        }
        of_group.x = wave_sum(of_group.x);
        of_group.y = wave_sum(of_group.y);
        if (lane == 0) group[sg] = make_float2(of_group.x * inv_m, of_group.y * inv_m);
    }
}

template <typename T, bool RAGGED, bool FROM_X> __global__ __launch_bounds__(GN_SPLIT_THREADS) void k_gn_backward_apply(GnBackwardArgs<T> a)
{
    const Slab& s = a.s;
    const int c = threadIdx.x % s.slots, pl = threadIdx.x / s.slots;
    for (int64_t turn = blockIdx.x; turn < 8 * s.per_xcd; turn += gridDim.x) {
        const int64_t item = item_of(s, turn);
        if (item < 0) continue;
        const int64_t sb = item / s.slices, sample = sb / a.blocks;
        const int slice = (int)(item - sb * s.slices), block = (int)(sb - sample * a.blocks);
        const int chunk = slice * s.slots + c, n = pl < s.lanes ? max(0, min(8, s.channels - 8 * chunk)) : 0;
        const int p0 = block * a.rows, pixels = min(a.rows, s.pixels - p0);
        const int64_t pixel0 = sample * s.pixels + p0;
        GnPixel<T, FROM_X> px[GN_APPLY_ROWS];
#pragma unroll
        for (int u = 0; u < GN_APPLY_ROWS; ++u) {
            const int p = pl + u * s.lanes;
            const bool there = n > 0 && p < pixels;
            load_pixel<T, RAGGED, FROM_X>(a, px[u], pixel0 + (there ? p : 0), chunk, there ? n : 0);
        }
        float w[8], b[8], m[8], rs[8], sg[8], sh[8];
        load_param<T>(a.weight, a.param_f32, 8 * (int64_t)chunk, n, 1.0f, w);
        load_param<T>(a.bias, a.param_f32, 8 * (int64_t)chunk, n, 0.0f, b);
        of_columns(8 * min(chunk, (s.channels - 1) / 8), s.d, s.groups, [&](int i, int g, int) {
            const int64_t from = sample * s.groups + g;
            m[i] = FROM_X ? a.mean[from] : 0.0f;
            rs[i] = a.rstd[from];
            const float2 t = a.group[from];
            sg[i] = t.x;
            sh[i] = t.y;
        });
        const float c2 = a.coeff ? 2.0f * a.coeff[sample] : 0.0f;
#pragma unroll
        for (int u = 0; u < GN_APPLY_ROWS; ++u) {
            const int p = pl + u * s.lanes;
            if (n > 0 && p < pixels) {
                float h[8], dz[8];
                dz_of(a, px[u], c2, m, rs, w, b, h, dz);
                store_dx<T, RAGGED>(a, pixel0 + p, chunk, n, h, dz, rs, w, sg, sh);
            }
        }
    }
}

// dgamma and dbeta: sums over the samples of a column's sums, sixteen columns to a workgroup, 64 threads to a column.
__global__ __launch_bounds__(1024) void k_gn_params(const float2* sums, int64_t samples, int32_t channels, float* dweight, float* dbias, int32_t accumulate)
{
    __shared__ float2 red[64][16];
    const int col = threadIdx.x & 15, lane = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
    float2 t = make_float2(0, 0);
    if (c < channels)
        for (int64_t b = lane; b < samples; b += 64) {
            const float2 v = sums[b * channels + c];
            t.x += v.x;
            t.y += v.y;
        }
    red[lane][col] = t;
    __syncthreads();
    for (int half = 32; half > 0; half >>= 1) {
        if (lane < half) {
            red[lane][col].x += red[lane + half][col].x;
            red[lane][col].y += red[lane + half][col].y;
        }
        __syncthreads();
    }
    if (lane == 0 && c < channels) {
        t = red[0][col];
        if (dweight) dweight[c] = accumulate ? dweight[c] + t.y : t.y;
        if (dbias) dbias[c] = accumulate ? dbias[c] + t.x : t.x;
    }
}

// ---- launches -------------------------------------------------------------------------------------------------------------
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
    s.cells_per_chunk = cells;
    s.parts = gn_parts(c.threads, c.slots, cells);
    s.items = samples * blocks * c.slices;
    s.per_xcd = (s.items + 7) / 8;
    return s;
}
static unsigned gn_grid(const Slab& s) { return (unsigned)std::min<int64_t>(8 * s.per_xcd, GN_MOST_GRID); }
static size_t lds_of(const GnCut& c, const Slab& s) { return gn_lds(c.threads, c.slots, s.cells_per_chunk, s.d); }

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

template <typename F> static hipError_t with_lds(F* kernel, size_t bytes)
{
    return bytes <= 65536 ? hipSuccess : hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}
#define GN_TRY(e) do { const hipError_t _e = (e); if (_e != hipSuccess) return _e; } while (0)

template <typename T, bool RAGGED, bool KEPT> static hipError_t gn_forward_of(const GroupNormForwardLaunch& f, hipStream_t s)
{
    constexpr int U = sizeof(T) == 4 ? 4 : 8;
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
        a.s = slab_of(p.cut, f.samples, f.pixels, f.channels, f.groups, 1, gn_cells(d, false));
        const size_t lds = lds_of(p.cut, a.s);
        if (p.cut.threads == 256) {
            GN_TRY(with_lds(k_gn_forward<T, RAGGED, KEPT, 256, U>, lds));
            k_gn_forward<T, RAGGED, KEPT, 256, U><<<gn_grid(a.s), 256, lds, s>>>(a);
        } else {
            GN_TRY(with_lds(k_gn_forward<T, RAGGED, KEPT, 1024, U>, lds));
            k_gn_forward<T, RAGGED, KEPT, 1024, U><<<gn_grid(a.s), 1024, lds, s>>>(a);
        }
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
        a.rows = p.stat.lanes * U;
        a.s = slab_of(p.stat, f.samples, f.pixels, f.channels, f.groups, p.blocks, p.pieces == 1 ? gn_cells(d, false) : 1);
        k_gn_stats<T, U><<<gn_grid(a.s), GN_SPLIT_THREADS, lds_of(p.stat, a.s), s>>>(a);
        GN_TRY(hipGetLastError());
        const int64_t all = f.samples * f.groups;
        k_gn_join<<<(unsigned)std::min<int64_t>((all + 3) / 4, GN_MOST_GRID), 256, 0, s>>>(part, stats, f.mean, f.rstd, all, p.pieces * p.blocks, f.eps);
        GN_TRY(hipGetLastError());
        a.good = f.goodness ? good : nullptr;
        a.blocks = p.apply_blocks;
        a.rows = p.cut.lanes * GN_APPLY_ROWS;
        a.s = slab_of(p.cut, f.samples, f.pixels, f.channels, f.groups, p.apply_blocks, 8);
        k_gn_apply<T, RAGGED, KEPT><<<gn_grid(a.s), GN_SPLIT_THREADS, 0, s>>>(a);
        GN_TRY(hipGetLastError());
    }
    if (f.goodness) k_gn_goodness<<<(unsigned)std::min<int64_t>((f.samples + 3) / 4, GN_MOST_GRID), 256, 0, s>>>(good, f.goodness, f.samples, parts);
    return hipGetLastError();
}
template <typename T> static hipError_t gn_forward_typed(const GroupNormForwardLaunch& f, hipStream_t s)
{
    const bool ragged = f.channels % 8 != 0;
    return f.q ? (ragged ? gn_forward_of<T, true, true>(f, s) : gn_forward_of<T, false, true>(f, s))
               : (ragged ? gn_forward_of<T, true, false>(f, s) : gn_forward_of<T, false, false>(f, s));
}
hipError_t launch_group_norm_forward(const GroupNormForwardLaunch& f, hipStream_t s)
{
    return f.dtype == FF_F32    ? gn_forward_typed<float>(f, s)
           : f.dtype == FF_BF16 ? gn_forward_typed<bf16_t>(f, s)
                                : gn_forward_typed<f16_t>(f, s);
}

static hipError_t launch_params(const float2* sums, const GroupNormBackwardLaunch& g, hipStream_t s)
{
    if (!g.dweight && !g.dbias) return hipSuccess;
    k_gn_params<<<(unsigned)((g.channels + 15) / 16), 1024, 0, s>>>(sums, g.samples, (int32_t)g.channels, g.dweight, g.dbias, g.accumulate);
    return hipGetLastError();
}
template <typename T, bool RAGGED, bool FROM_X> static hipError_t gn_backward_of(const GroupNormBackwardLaunch& g, hipStream_t s)
{
    constexpr int U = sizeof(T) == 4 ? 2 : 4;
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
    a.act = g.act;
    a.param_f32 = g.param_dtype == FF_F32;
    a.inv_m = (float)(1.0 / ((double)g.pixels * (double)d));
    if (!FROM_X) a.k = ckpt_ptr(g.q, g.e, g.channels);
    const bool params = g.dweight || g.dbias;
    float2* const sums = (float2*)g.ws;   // of every sample's columns
    if (p.whole) {
        a.sums = params ? sums : nullptr;
        a.s = slab_of(p.cut, g.samples, g.pixels, g.channels, g.groups, 1, 8);
        const size_t lds = lds_of(p.cut, a.s);
        if (p.cut.threads == 256) {
            GN_TRY(with_lds(k_gn_backward<T, RAGGED, FROM_X, 256, U>, lds));
            k_gn_backward<T, RAGGED, FROM_X, 256, U><<<gn_grid(a.s), 256, lds, s>>>(a);
        } else {
            GN_TRY(with_lds(k_gn_backward<T, RAGGED, FROM_X, 1024, U>, lds));
            k_gn_backward<T, RAGGED, FROM_X, 1024, U><<<gn_grid(a.s), 1024, lds, s>>>(a);
        }
        GN_TRY(hipGetLastError());
    } else {
        float2* const part = sums + g.samples * g.channels;
        float2* const group = part + g.samples * g.channels * p.blocks;
        a.sums = part;
        a.blocks = p.blocks;
        a.rows = (int32_t)((g.pixels + p.blocks - 1) / p.blocks);
        a.s = slab_of(p.stat, g.samples, g.pixels, g.channels, g.groups, p.blocks, 8);
        k_gn_backward_sums<T, RAGGED, FROM_X><<<gn_grid(a.s), GN_SPLIT_THREADS, lds_of(p.stat, a.s), s>>>(a);
        GN_TRY(hipGetLastError());
        const int64_t all = g.samples * g.groups;
        k_gn_backward_join<T><<<(unsigned)std::min<int64_t>((all + 3) / 4, GN_MOST_GRID), 256, 0, s>>>(part, sums, group, g.weight, a.param_f32, g.samples,
                                                                                                (int32_t)g.groups, (int32_t)d, p.blocks, a.inv_m);
        GN_TRY(hipGetLastError());
        if (g.dx) {
            a.group = group;
            a.blocks = p.apply_blocks;
            a.rows = p.cut.lanes * GN_APPLY_ROWS;
            a.s = slab_of(p.cut, g.samples, g.pixels, g.channels, g.groups, p.apply_blocks, 8);
            k_gn_backward_apply<T, RAGGED, FROM_X><<<gn_grid(a.s), GN_SPLIT_THREADS, 0, s>>>(a);
            GN_TRY(hipGetLastError());
        }
    }
    return launch_params(sums, g, s);
}
template <typename T> static hipError_t gn_backward_typed(const GroupNormBackwardLaunch& g, hipStream_t s)
{
    const bool ragged = g.channels % 8 != 0;
    return g.x ? (ragged ? gn_backward_of<T, true, true>(g, s) : gn_backward_of<T, false, true>(g, s))
               : (ragged ? gn_backward_of<T, true, false>(g, s) : gn_backward_of<T, false, false>(g, s));
}
hipError_t launch_group_norm_backward(const GroupNormBackwardLaunch& g, hipStream_t s)
{
    if (g.samples == 0) return launch_params((const float2*)g.ws, g, s);
    return g.dtype == FF_F32    ? gn_backward_typed<float>(g, s)
           : g.dtype == FF_BF16 ? gn_backward_typed<bf16_t>(g, s)
                                : gn_backward_typed<f16_t>(g, s);
}

}  // namespace ffi
