// Layer norm, forward and backward, over the rows of a matrix of fp32, bf16 or fp16 values.
//
//   mean = 1/C sum x,  rstd = 1 / sqrt(1/C sum (x - mean)^2 + eps),  h = (x - mean) rstd,  y = h w + b
//   g = dy w,  dx = rstd (g - 1/C sum g - h 1/C sum g h),  dw = sum over rows of dy h,  db = sum over rows of dy
//
// Statistics, products and sums are fp32; y and dx are rounded once.  The forward pass sums a row, and then, over values that are held in registers, the
// deviations from that mean and their squares: what is left of the mean, 1/C of the deviations' sum, is taken out of the mean, every deviation and the variance.
// Without it a mean's rounding goes into all of a row's h, which the checkpoint scales up where they are small: 500 values of 1000.0 gave h = -0.02 each, and give 0.
// That is for rows farther from zero than they are wide.  There the deviations are exact or nearly; elsewhere their own roundings are more than what the first sum
// lacks, and the mean stays as it is.
//
// Both are bound by memory: a row is read once and held in registers by a group of 4 to 1024 lanes, eight columns (a chunk) of a lane
// at a time.  The forward pass can write the checkpoint of h beside y, and the backward pass reads h from it (1.03 bytes a value) instead of x.
//
// Measured, us and TB/s, inputs from memory (a copy of as many bytes reaches 5.3):
//                                    16384 x 4096 bf16    16384 x 4096 fp32    131072 x 784 bf16    262144 x 128 fp16
//   forward                              51   5.2              99   5.4              83   4.9              29   4.6
//   forward, codes to nearest            67   5.0             114   5.3             111   4.7              40   4.3
//   forward, stochastic codes         72-76   4.5             116   5.2             129   4.0              51   3.3
//   backward from x                      80   5.0             159   5.1             146   4.2              50   4.0
//   backward from the checkpoint         70   4.8             118   5.1             136   3.8              41   4.2
// Stochastic codes of 16-bit values are as much arithmetic as memory: 38 operations a value, of which the random word takes ten.  784 columns are 98 chunks on
// 64 lanes with two each: a quarter of what is issued works on columns that do not exist.
#include <type_traits>

#include "ckpt.hpp"
#include "norm.hpp"

namespace ffi {

template <int LANES> struct Group {
    static constexpr int THREADS = LANES <= 64 ? 256 : LANES;
    static constexpr int ROWS = THREADS / LANES;   // groups of a workgroup
    // a lane's group; where a wavefront has one only, a scalar, and with it all addresses of its row
    static __device__ __forceinline__ int mine()
    {
        if constexpr (ROWS == 1) return 0;
        else if constexpr (LANES == 64) return __builtin_amdgcn_readfirstlane(threadIdx.x / LANES);
        else return threadIdx.x / LANES;
    }
};

// Sum over the lanes of a group, which every lane receives.  Groups of more than a wavefront meet in `red`, one word per wavefront
// and sum, which the caller does not use twice between barriers.
template <int LANES, int N> __device__ __forceinline__ void group_sum(float (&v)[N], float* red)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        auto add = [&](auto ctrl) { v[i] += __uint_as_float(dpp_u32<decltype(ctrl)::value>(__float_as_uint(v[i]))); };
        add(std::integral_constant<int, 0xB1>());                                  // quad_perm [1,0,3,2]
        add(std::integral_constant<int, 0x4E>());                                  // quad_perm [2,3,0,1]
        if constexpr (LANES >= 8) add(std::integral_constant<int, 0x141>());       // row_half_mirror
        if constexpr (LANES >= 16) add(std::integral_constant<int, 0x140>());      // row_mirror
        if constexpr (LANES >= 32) v[i] += __shfl_xor(v[i], 16);
        if constexpr (LANES >= 64) v[i] += __shfl_xor(v[i], 32);
    }
    if constexpr (LANES > 64) {
        constexpr int W = LANES / 64;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) red[i * W + wave] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float t = 0;
#pragma unroll
            for (int w = 0; w < W; ++w) t += red[i * W + w];
            v[i] = t;
        }
    }
}

// 1 / sqrt(v) to one unit in the last place; the instruction takes no numbers below 2^-126.
__device__ __forceinline__ float inverse_root(float v)
{
    const bool low = v < 0x1p-96f;
    const float r = __builtin_amdgcn_rsqf(low ? v * 0x1p96f : v);
    return low ? r * 0x1p48f : r;
}

// What is left of a row's mean, by the mean of the deviations from it and that of their squares; and the variance.  (Not below zero by a rounding; NaN stays.)
__device__ __forceinline__ float mean_rest(float mean, float deviation, float square) { return mean * mean > square ? deviation : 0.0f; }
__device__ __forceinline__ float variance(float square, float rest)
{
    const float v = __builtin_fmaf(-rest, rest, square);
    return v < 0 ? 0.0f : v;
}

// Eight parameters of a chunk (n of them exist), in the element's type or in fp32; `none` where there are none.
template <typename T> __device__ __forceinline__ void load_param(const void* p, bool f32, int64_t at, int n, float none, float v[8])
{
    if (p == nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = none;
    } else if (sizeof(T) == 4 || f32) {
        load8((const float*)p + at, n, v);
    } else {
        load8((const T*)p + at, n, v);
    }
}

template <int LANES> constexpr RowEnds row_ends(bool ragged) { return !ragged ? ROWS_WHOLE : LANES == 4 ? ROWS_ANY : ROWS_RAGGED; }
template <bool RAGGED, typename T> __device__ __forceinline__ void row_store(T* row, int c, int n, const float v[8])
{
    if constexpr (RAGGED) store8(row + 8 * c, n, v);
    else if (n > 0) store8(row + 8 * c, 8, v);
}

template <typename T> struct NormForwardArgs {
    const T* x;
    T* y;
    int64_t ldx, ldy, rows;
    const void* weight;
    const void* bias;
    float* mean;
    float* rstd;
    int32_t cols, param_f32;
    float eps, inv_cols;
    CkptPtr k;
    CkptRound r;
};

// Groups that take row after row.  (Up to 64 chunks to a row, the next group's wavefronts hide as much: 65536 x 512 fp32 42 us, and 48 row after
// row.  Four chunks of 1024 lanes leave no registers to spare.)
constexpr bool many_rows(int lanes, int ch) { return lanes * ch > 64 && lanes * ch < 4096; }

// CH chunks of a lane.  Groups that take row after row keep the parameters in registers and have the next row's values on their way; the others take
// one row each, whose few parameters the cache holds.
template <typename T, int LANES, int CH, bool RAGGED>
__global__ __launch_bounds__(Group<LANES>::THREADS) void k_norm_forward(NormForwardArgs<T> a)
{
    constexpr int W = LANES > 64 ? LANES / 64 : 1;
    constexpr bool MANY = many_rows(LANES, CH);
    __shared__ float red[3 * W];   // the first sum's words, the second's (written again behind the other sum's barrier)
    const int j = threadIdx.x % LANES;
    const int64_t first = (int64_t)blockIdx.x * Group<LANES>::ROWS;   // the workgroup's; `row` is that, or the wavefront's, and r the group's row behind it
    const int64_t row0 = first + Group<LANES>::mine();
    if (LANES == 64 && row0 >= a.rows) return;   // (a whole wavefront, which meets no other)
    const bool there = Group<LANES>::ROWS == 1 || LANES == 64 || row0 < a.rows;   // (lanes of a row that does not exist go along and store nothing)
    int cols = a.cols;
    auto count = [&](int i) { return max(0, min(8, cols - 8 * (j + i * LANES))); };
    Raw8<T> raw[CH];
    int64_t row = LANES < 64 ? first : row0;
    const uint32_t r = LANES < 64 && there ? Group<LANES>::mine() : 0;
    auto fetch = [&](int64_t row) {
        const T* const x = element(a.x, a.ldx, row, r, 0);
#pragma unroll
        for (int i = 0; i < CH; ++i) raw[i] = row_chunk<row_ends<LANES>(RAGGED)>(x, j + i * LANES, count(i), cols);
    };
    fetch(row);
    float w[MANY ? CH : 1][8], b[MANY ? CH : 1][8];
    auto params = [&](int i, float* w, float* b) {
        load_param<T>(a.weight, a.param_f32, 8 * (j + i * LANES), count(i), 1.0f, w);
        load_param<T>(a.bias, a.param_f32, 8 * (j + i * LANES), count(i), 0.0f, b);
    };
    if constexpr (MANY)
#pragma unroll
        for (int i = 0; i < CH; ++i) params(i, w[i], b[i]);
    for (;;) {
        opaque_uniform(cols);   // (the masks of all chunks, kept from row to row, are more than there are scalar registers)
        float v[CH][8], sum[1] = {0};
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            settle<row_ends<LANES>(RAGGED)>(raw[i], count(i), cols);
            raw_values(raw[i], v[i]);
#pragma unroll
            for (int u = 0; u < 8; ++u) sum[0] += v[i][u];
        }
        const int64_t next = row + (int64_t)gridDim.x * Group<LANES>::ROWS;
        if (MANY && next < a.rows) fetch(next);
        group_sum<LANES, 1>(sum, red);
        const float mean = sum[0] * a.inv_cols;
        float dev[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int n = count(i);
            if (n < 8) {   // columns that do not exist lie at the mean from here on
#pragma unroll
                for (int u = 0; u < 8; ++u) v[i][u] = RAGGED && u < n ? v[i][u] : mean;
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                v[i][u] -= mean;
                dev[0] += v[i][u];
                dev[1] = __builtin_fmaf(v[i][u], v[i][u], dev[1]);
            }
        }
        group_sum<LANES, 2>(dev, red + W);
        const float square = dev[1] * a.inv_cols, rest = mean_rest(mean, dev[0] * a.inv_cols, square);
        const float rstd = inverse_root(variance(square, rest) + a.eps), shift = -rest * rstd;
        if (there && j == 0) {
            if (a.mean) a.mean[row + r] = mean + rest;
            if (a.rstd) a.rstd[row + r] = rstd;
        }
        T* const y = element(a.y, a.ldy, row, r, 0);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            opaque_uniform(cols);
            const int c = j + i * LANES, n = count(i);
            float h[8], o[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) h[u] = __builtin_fmaf(v[i][u], rstd, shift);
            if constexpr (!MANY) params(i, w[0], b[0]);
#pragma unroll
            for (int u = 0; u < 8; ++u) o[u] = __builtin_fmaf(h[u], w[MANY ? i : 0][u], b[MANY ? i : 0][u]);
            row_store<RAGGED>(y, c, there ? n : 0, o);
            if (a.k.q) {
                if (RAGGED && n < 8) {   // columns that do not exist are nothing to a block's largest value
#pragma unroll
                    for (int u = 0; u < 8; ++u) h[u] = u < n ? h[u] : 0.0f;
                }
                const uint32_t m = quad_max_u32(RAGGED || n > 0 ? abs_max_bits(h) : 0u), e = ckpt_exponent(m);
                const u32x2 q = ckpt_codes(h, m, e, a.r, (uint64_t)row * (uint64_t)a.cols + ((uint64_t)r * (uint32_t)a.cols + 8 * (uint32_t)c));
                if (there)
                    ckpt_store_chunk(a.k, element(a.k.q, a.k.pitch, row, r, 0), element(a.k.e, a.k.epitch, row, r, 0), c, LANES * CH, n > 0, q, e);
            }
        }
        if (!MANY || next >= a.rows) break;
        row = next;
    }
}

// Rows of more columns than a workgroup holds (32768): read three times, from the caches but for the first.
template <typename T> __global__ __launch_bounds__(1024) void k_norm_forward_wide(NormForwardArgs<T> a)
{
    __shared__ float red[3 * 16];
    const int64_t row = blockIdx.x;
    const T* const x = a.x + row * a.ldx;
    T* const y = a.y + row * a.ldy;
    const int chunks = (int)(a.k.pitch / 8 + 1023) / 1024 * 1024;   // (pad columns of the checkpoint included, whole wavefronts)
    float sum[1] = {0};
    for (int c = threadIdx.x; c < chunks; c += 1024) {
        float v[8];
        load8(x + 8 * c, max(0, min(8, a.cols - 8 * c)), v);
#pragma unroll
        for (int u = 0; u < 8; ++u) sum[0] += v[u];
    }
    group_sum<1024, 1>(sum, red);
    const float mean = sum[0] * a.inv_cols;
    auto deviations = [&](int c, float v[8]) {
        const int n = max(0, min(8, a.cols - 8 * c));
        load8(x + 8 * c, n, v);
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = u < n ? v[u] - mean : 0.0f;
        return n;
    };
    float dev[2] = {0, 0};
    for (int c = threadIdx.x; c < chunks; c += 1024) {
        float v[8];
        deviations(c, v);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            dev[0] += v[u];
            dev[1] = __builtin_fmaf(v[u], v[u], dev[1]);
        }
    }
    group_sum<1024, 2>(dev, red + 16);
    const float square = dev[1] * a.inv_cols, rest = mean_rest(mean, dev[0] * a.inv_cols, square);
    const float rstd = inverse_root(variance(square, rest) + a.eps), shift = -rest * rstd;
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mean + rest;
        if (a.rstd) a.rstd[row] = rstd;
    }
    for (int c = threadIdx.x; c < chunks; c += 1024) {
        float h[8], w[8], b[8], o[8];
        const int n = deviations(c, h);
        load_param<T>(a.weight, a.param_f32, 8 * c, n, 1.0f, w);
        load_param<T>(a.bias, a.param_f32, 8 * c, n, 0.0f, b);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            h[u] = u < n ? __builtin_fmaf(h[u], rstd, shift) : 0.0f;
            o[u] = __builtin_fmaf(h[u], w[u], b[u]);
        }
        store8(y + 8 * c, n, o);
        if (a.k.q) {
            const uint32_t m = quad_max_u32(abs_max_bits(h)), e = ckpt_exponent(m);
            const u32x2 q = ckpt_codes(h, m, e, a.r, (uint64_t)row * (uint64_t)a.cols + 8 * (uint64_t)c);
            ckpt_store_chunk(a.k, a.k.q + row * a.k.pitch, a.k.e + row * a.k.epitch, c, chunks, n > 0, q, e);
        }
    }
}

// ------------------------------------------------------------------------------------------------
// Backward.  A workgroup keeps the column sums of its rows in registers (a lane's columns never change) and leaves them in the
// workspace; k_norm_columns adds the workgroups' sums in order, so results do not depend on timing.  Of few rows, other workgroups of the same launch
// make the column sums (of a launch of their own, before it, where dx overwrites what they read).
// ------------------------------------------------------------------------------------------------
template <typename T> struct NormBackwardArgs {
    const T* dy;
    const T* x;
    T* dx;
    int64_t lddy, ldx, lddx, rows;
    const float* mean;
    const float* rstd;
    const void* weight;
    int32_t cols, param_f32, sums;   // sums: dweight or dbias is wanted
    float inv_cols;
    CkptPtr k;
    float* part;        // [workgroups][2][pcols]
    int64_t pcols;
    float2* row_sums;   // rows too wide for registers: both means of every row
    int64_t row_wgs;    // workgroups that take rows; those behind them take columns, and leave dweight and dbias
    float* dweight;
    float* dbias;
    int32_t accumulate;
};

// Few rows: 64 columns of all of them and their sums, while other workgroups work on dx.  What is read twice costs less than a second launch.
// lds: sixteen words a thread.
template <typename T, bool KEPT, int THREADS> __device__ __forceinline__ void column_sums(const NormBackwardArgs<T>& a, int64_t part, float* lds)
{
    constexpr int S = THREADS / 8;
    const int lane = threadIdx.x & 7, slice = threadIdx.x >> 3, first = (int)part * 64, at = first + 8 * lane, n = max(0, min(8, a.cols - at));
    float dw[8], db[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) dw[u] = db[u] = 0;
    if (n > 0) {
#pragma unroll 4
        for (int64_t row = slice; row < a.rows; row += S) {
            float d[8], h[8];
            load8(a.dy + row * a.lddy + at, n, d);
            if constexpr (KEPT) {
                ckpt_values(*(const u32x2*)(a.k.q + row * a.k.pitch + at), a.k.e[row * a.k.epitch + (at >> 5)], h);
            } else {
                const float rstd = a.rstd[row], mean = a.mean[row];
                load8(a.x + row * a.ldx + at, n, h);
#pragma unroll
                for (int u = 0; u < 8; ++u) h[u] = (h[u] - mean) * rstd;
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                dw[u] = __builtin_fmaf(d[u], h[u], dw[u]);
                db[u] += d[u];
            }
        }
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        lds[threadIdx.x * 16 + u] = dw[u];
        lds[threadIdx.x * 16 + 8 + u] = db[u];
    }
    __syncthreads();
    const int col = threadIdx.x & 63;
    float* const out = threadIdx.x < 64 ? a.dweight : a.dbias;
    if (threadIdx.x >= 128 || first + col >= a.cols || !out) return;
    const float* const from = lds + (col >> 3) * 16 + (threadIdx.x >> 6) * 8 + (col & 7);
    float v = 0;
#pragma unroll 8
    for (int s = 0; s < S; ++s) v += from[s * 128];
    out[first + col] = a.accumulate ? out[first + col] + v : v;
}

// Rows of a group in a round; the next round's are on their way meanwhile.
template <typename T, int CH> constexpr int rows_ahead() { return sizeof(T) == 4 || CH > 1 ? 1 : 2; }

template <typename T, bool KEPT, int LANES, int CH, bool RAGGED>
__global__ __launch_bounds__(Group<LANES>::THREADS) void k_norm_backward(NormBackwardArgs<T> a)
{
    using G = Group<LANES>;
    constexpr int W = LANES > 64 ? LANES / 64 : 1, R = rows_ahead<T, CH>();
    __shared__ float red[2][2 * R * W];
    __shared__ __attribute__((aligned(16))) float cols_lds[G::THREADS * 16];
    if (blockIdx.x >= a.row_wgs) {
        column_sums<T, KEPT, G::THREADS>(a, blockIdx.x - a.row_wgs, cols_lds);
        return;
    }
    const int j = threadIdx.x % LANES, group = G::mine();
    const int64_t groups = a.row_wgs * G::ROWS, g0 = (int64_t)blockIdx.x * G::ROWS + group;
    int cols = a.cols;
    auto count = [&](int i) { return max(0, min(8, cols - 8 * (j + i * LANES))); };
    // The weight is held in registers, or, where a lane has four chunks, in LDS: in memory its loads would wait for the next rows'.
    constexpr bool HELD = CH < 4;
    __shared__ __attribute__((aligned(16))) float w_lds[HELD ? 4 : LANES * CH * 8];
    float held[HELD ? CH : 1][8], dw[CH][8], db[CH][8];
    typedef float f32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int i = 0; i < CH; ++i) {
#pragma unroll
        for (int u = 0; u < 8; ++u) dw[i][u] = db[i][u] = 0;
        float* const w = held[HELD ? i : 0];
        load_param<T>(a.weight, a.param_f32, 8 * (j + i * LANES), count(i), 1.0f, w);
        if constexpr (!HELD) {   // (two planes of four floats a lane: neighbouring lanes in neighbouring banks)
            ((f32x4*)w_lds)[(2 * i) * LANES + j] = f32x4{w[0], w[1], w[2], w[3]};
            ((f32x4*)w_lds)[(2 * i + 1) * LANES + j] = f32x4{w[4], w[5], w[6], w[7]};
        }
    }
    auto weight = [&](int i, float w[8]) {   // (a lane reads what it wrote)
        if constexpr (HELD) {
#pragma unroll
            for (int u = 0; u < 8; ++u) w[u] = held[i][u];
        } else {
            const f32x4 lo = ((const f32x4*)w_lds)[(2 * i) * LANES + j], hi = ((const f32x4*)w_lds)[(2 * i + 1) * LANES + j];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                w[u] = lo[u];
                w[4 + u] = hi[u];
            }
        }
    };
    struct Rows {
        Raw8<T> d[R][CH];
        std::conditional_t<KEPT, u32x2, Raw8<T>> x[R][CH];
        uint32_t e[R][CH];
        float mean[R], rstd[R];
    };
    // Row k of round `it`, as a scalar and what a lane's group adds to it; one that does not exist is some other, with zeros for everything.
    const uint32_t own = LANES < 64 ? group : 0;
    const int64_t base = LANES < 64 ? (int64_t)blockIdx.x * G::ROWS : g0;
    auto row_of = [&](int64_t it, int k) { return (it * R + k) * groups + base; };
    auto fetch = [&](int64_t it, Rows& to) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const bool there = row_of(it, k) + own < a.rows;
            const int64_t row = min(row_of(it, k), a.rows - 1);
            const uint32_t r = there ? own : 0;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int c = j + i * LANES, n = there ? count(i) : 0;
                if constexpr (KEPT) {
                    const int at = n > 0 ? c : 0;
                    const u32x2 q = *(const u32x2*)element(a.k.q, a.k.pitch, row, r, 8 * at);
                    const uint32_t e = *element(a.k.e, a.k.epitch, row, r, at >> 2);
                    to.x[k][i] = n > 0 ? q : u32x2{0, 0};
                    to.e[k][i] = n > 0 ? e : 127u;
                } else {
                    to.x[k][i] = row_chunk<row_ends<LANES>(RAGGED)>(element(a.x, a.ldx, row, r, 0), c, n, cols);
                    to.e[k][i] = 0;
                }
                to.d[k][i] = row_chunk<row_ends<LANES>(RAGGED)>(element(a.dy, a.lddy, row, r, 0), c, n, cols);
            }
            const float rstd = a.rstd[row + r], mean = KEPT ? 0.0f : a.mean[row + r];
            to.rstd[k] = there ? rstd : 0.0f;
            to.mean[k] = there ? mean : 0.0f;
        }
    };
    auto values = [&](const Rows& r, int k, int i, float d[8], float h[8]) {
        raw_values(r.d[k][i], d);
        if constexpr (KEPT) {
            ckpt_values(r.x[k][i], r.e[k][i], h);
        } else {
            raw_values(r.x[k][i], h);
#pragma unroll
            for (int u = 0; u < 8; ++u) h[u] = (h[u] - r.mean[k]) * r.rstd[k];
        }
    };
    // every group of a workgroup of several wavefronts makes the same number of rounds: barriers are inside
    const int64_t rounds = (a.rows + groups * R - 1) / (groups * R);
    constexpr bool AHEAD = CH < 4 || (sizeof(T) == 2 && (KEPT || !RAGGED));   // (the others of four chunks have no registers for a second row)
    Rows now, next;
    if constexpr (AHEAD) fetch(0, next);
    for (int64_t it = 0; it < rounds; ++it) {
        opaque_uniform(cols);   // (see k_norm_forward)
        if constexpr (AHEAD) {
            now = next;
            fetch(min(it + 1, rounds - 1), next);
        } else {
            fetch(it, now);
        }
        float s[2 * R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            s[2 * k] = s[2 * k + 1] = 0;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                // (a column that does not exist has d = 0 and adds nothing, or a NaN where the row's own columns have them too)
                float d[8], h[8], w[8];
                const int n = row_of(it, k) + own < a.rows ? count(i) : 0;
                settle<row_ends<LANES>(RAGGED)>(now.d[k][i], n, cols);
                if constexpr (!KEPT) settle<row_ends<LANES>(RAGGED)>(now.x[k][i], n, cols);
                values(now, k, i, d, h);
                weight(i, w);
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const float g = d[u] * w[u];
                    s[2 * k] += g;
                    s[2 * k + 1] = __builtin_fmaf(g, h[u], s[2 * k + 1]);
                    dw[i][u] = __builtin_fmaf(d[u], h[u], dw[i][u]);
                    db[i][u] += d[u];
                }
                if constexpr (CH == 4) __builtin_amdgcn_sched_barrier(0);   // (chunk by chunk: registers)
            }
        }
        if (a.dx) {
            group_sum<LANES, 2 * R>(s, red[it & 1]);
#pragma unroll
            for (int k = 0; k < R; ++k)
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    opaque(now.d[k][i]);
                    opaque(now.x[k][i]);
                }
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const float c1 = s[2 * k] * a.inv_cols, c2 = s[2 * k + 1] * a.inv_cols;
                const int64_t row = row_of(it, k);
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    float d[8], h[8], w[8];
                    values(now, k, i, d, h);
                    weight(i, w);
#pragma unroll
                    for (int u = 0; u < 8; ++u) d[u] = now.rstd[k] * (d[u] * w[u] - c1 - h[u] * c2);
                    row_store<RAGGED>(element(a.dx, a.lddx, row, own, 0), j + i * LANES, row + own < a.rows ? count(i) : 0, d);
                    if constexpr (CH == 4) __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    }
    if (!a.sums) return;
    float* const out = a.part + (int64_t)blockIdx.x * 2 * a.pcols;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = j + i * LANES;
        if constexpr (G::ROWS > 1) {   // the workgroup's groups hold the same columns: sixteen words a lane, added in order
            float* const mine = cols_lds + threadIdx.x * 16;
            __syncthreads();
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                mine[u] = dw[i][u];
                mine[8 + u] = db[i][u];
            }
            __syncthreads();
            for (int t = threadIdx.x; t < LANES * 16; t += G::THREADS) {
                float v = 0;
#pragma unroll 4
                for (int g = 0; g < G::ROWS; ++g) v += cols_lds[g * LANES * 16 + t];
                const int64_t col = 8 * (int64_t)(t / 16 + i * LANES) + (t & 7);
                if (col < a.pcols) out[((t >> 3) & 1) * a.pcols + col] = v;
            }
        } else if (8 * c < a.pcols) {
#pragma unroll
            for (int u = 0; u < 8; u += 4) {
                *(float4*)(out + 8 * c + u) = make_float4(dw[i][u], dw[i][u + 1], dw[i][u + 2], dw[i][u + 3]);
                *(float4*)(out + a.pcols + 8 * c + u) = make_float4(db[i][u], db[i][u + 1], db[i][u + 2], db[i][u + 3]);
            }
        }
    }
}

// Rows of more columns than a workgroup holds: their two means first, ...
template <typename T, bool KEPT> __global__ __launch_bounds__(1024) void k_norm_row_sums(NormBackwardArgs<T> a)
{
    __shared__ float red[2 * 16];
    const int64_t row = blockIdx.x;
    float s[2] = {0, 0};
    const float rstd = a.rstd[row], mean = KEPT ? 0.0f : a.mean[row];
    for (int c = threadIdx.x; 8 * c < a.cols; c += 1024) {
        const int n = min(8, a.cols - 8 * c);
        float d[8], h[8], w[8];
        load8(a.dy + row * a.lddy + 8 * c, n, d);
        if constexpr (KEPT) {
            ckpt_values(*(const u32x2*)(a.k.q + row * a.k.pitch + 8 * c), a.k.e[row * a.k.epitch + (c >> 2)], h);
        } else {
            load8(a.x + row * a.ldx + 8 * c, n, h);
#pragma unroll
            for (int u = 0; u < 8; ++u) h[u] = (h[u] - mean) * rstd;
        }
        load_param<T>(a.weight, a.param_f32, 8 * c, n, 1.0f, w);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float g = d[u] * w[u];
            s[0] += g;
            s[1] = __builtin_fmaf(g, h[u], s[1]);
        }
    }
    group_sum<1024, 2>(s, red);
    if (threadIdx.x == 0) a.row_sums[row] = make_float2(s[0] * a.inv_cols, s[1] * a.inv_cols);
}
// ... then dx and the column sums of 2048 columns and every gridDim.y-th row.
template <typename T, bool KEPT> __global__ __launch_bounds__(256) void k_norm_backward_wide(NormBackwardArgs<T> a)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    const int n = min(8, a.cols - 8 * c);
    if (n <= 0) return;
    float w[8], dw[8], db[8];
    load_param<T>(a.weight, a.param_f32, 8 * c, n, 1.0f, w);
#pragma unroll
    for (int u = 0; u < 8; ++u) dw[u] = db[u] = 0;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float rstd = a.rstd[row], mean = KEPT ? 0.0f : a.mean[row];
        float d[8], h[8];
        load8(a.dy + row * a.lddy + 8 * c, n, d);
        if constexpr (KEPT) {
            ckpt_values(*(const u32x2*)(a.k.q + row * a.k.pitch + 8 * c), a.k.e[row * a.k.epitch + (c >> 2)], h);
        } else {
            load8(a.x + row * a.ldx + 8 * c, n, h);
#pragma unroll
            for (int u = 0; u < 8; ++u) h[u] = (h[u] - mean) * rstd;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            dw[u] = __builtin_fmaf(d[u], h[u], dw[u]);
            db[u] += d[u];
        }
        if (a.dx) {
            const float2 m = a.row_sums[row];
#pragma unroll
            for (int u = 0; u < 8; ++u) d[u] = rstd * (d[u] * w[u] - m.x - h[u] * m.y);
            store8(a.dx + row * a.lddx + 8 * c, n, d);
        }
    }
    if (!a.sums) return;
    float* const out = a.part + (int64_t)blockIdx.y * 2 * a.pcols + 8 * c;   // (pcols is a multiple of eight)
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        out[u] = dw[u];
        out[a.pcols + u] = db[u];
    }
}

// Adds the workgroups' column sums: 32 columns (a cache line of fp32) by 64 slices of the workgroups, then the slices in order.
__global__ __launch_bounds__(512) void k_norm_columns(const float* part, int parts, int64_t pcols, int cols, float* dw, float* db, int accumulate)
{
    __shared__ float red[64][33], last[16][32];
    const int lane = threadIdx.x & 7, slice = threadIdx.x >> 3, col = blockIdx.x * 32;
    float* const out = blockIdx.y ? db : dw;
    if (!out) return;
    float4 v = make_float4(0, 0, 0, 0);
    if (col + 4 * lane < pcols) {   // (pcols is a multiple of eight)
        const float* const p = part + blockIdx.y * pcols + col + 4 * lane;
#pragma unroll 8
        for (int g = slice; g < parts; g += 64) {
            const float4 t = *(const float4*)(p + (int64_t)g * 2 * pcols);
            v = make_float4(v.x + t.x, v.y + t.y, v.z + t.z, v.w + t.w);
        }
    }
    red[slice][4 * lane] = v.x;
    red[slice][4 * lane + 1] = v.y;
    red[slice][4 * lane + 2] = v.z;
    red[slice][4 * lane + 3] = v.w;
    __syncthreads();
    const int c = threadIdx.x & 31, q = threadIdx.x >> 5;
    last[q][c] = (red[4 * q][c] + red[4 * q + 1][c]) + (red[4 * q + 2][c] + red[4 * q + 3][c]);
    __syncthreads();
    if (threadIdx.x < 32 && col + c < cols) {
        float sum = 0;
#pragma unroll
        for (int g = 0; g < 16; ++g) sum += last[g][c];
        out[col + c] = accumulate ? out[col + c] + sum : sum;
    }
}

// ------------------------------------------------------------------------------------------------
// launches
// ------------------------------------------------------------------------------------------------
template <typename T, int LANES, int CH> static hipError_t forward_as(const NormForwardArgs<T>& a, hipStream_t s)
{
    // row after row: as many workgroups as run at once (16384 x 4096 bf16 with stochastic codes, both before the codes' arithmetic was cut: 97 us with one
    // row each, 80 row after row)
    const int64_t wgs = (a.rows + Group<LANES>::ROWS - 1) / Group<LANES>::ROWS, most = many_rows(LANES, CH) ? 256 * (1024 / Group<LANES>::THREADS) : wgs;
    const dim3 grid((unsigned)min(wgs, most));
    if (a.cols % 8 == 0) k_norm_forward<T, LANES, CH, false><<<grid, Group<LANES>::THREADS, 0, s>>>(a);
    else k_norm_forward<T, LANES, CH, true><<<grid, Group<LANES>::THREADS, 0, s>>>(a);
    return hipGetLastError();
}
template <typename T> static hipError_t forward_of(const NormForwardLaunch& l, hipStream_t s)
{
    NormForwardArgs<T> a;
    a.x = (const T*)l.x;
    a.y = (T*)l.y;
    a.ldx = l.ldx;
    a.ldy = l.ldy;
    a.rows = l.rows;
    a.weight = l.weight;
    a.bias = l.bias;
    a.mean = l.mean;
    a.rstd = l.rstd;
    a.cols = (int32_t)l.cols;
    a.param_f32 = l.param_dtype == FF_F32;
    a.eps = l.eps;
    a.inv_cols = 1.0f / (float)l.cols;
    a.k = ckpt_ptr(l.q, l.e, l.cols);
    a.r = {make_sr_key(l.seed, l.tag), l.round_mode == FF_ROUND_STOCHASTIC};
    // Lanes of a row: as few as hold it in two chunks each, since a wavefront's own sums need no barrier and fewer lanes are left over (131072 x 784
    // bf16, stochastic codes: 359 us by 256 lanes with a chunk each, 129 by 64; 32768 x 2000: 101 by 256, 74 by 128), and the smallest power of two for
    // one chunk below that.  (Of few rows one chunk a lane, half as many rows at once, is faster: 512 x 784 fp32 3.7 us by this and 3.4 by 128 lanes, 64 x 1001
    // bf16 with stochastic codes 4.8 and 3.7, 1024 x 2000 fp32 5.4 and 5.3; 2048 x 2000 8.9 both with codes to nearest, 9.2 and 10.7 with stochastic ones.
    // The rows are not asked.)
    const int64_t chunks = (a.k.pitch / 8 + 3) / 4 * 4;   // (pad columns of the checkpoint included)
    if (chunks <= 4) return forward_as<T, 4, 1>(a, s);
    if (chunks <= 8) return forward_as<T, 8, 1>(a, s);
    if (chunks <= 16) return forward_as<T, 16, 1>(a, s);
    if (chunks <= 32) return forward_as<T, 32, 1>(a, s);
    if (chunks <= 64) return forward_as<T, 64, 1>(a, s);
    if (chunks <= 128) return forward_as<T, 64, 2>(a, s);
    if (chunks <= 256) return forward_as<T, 128, 2>(a, s);
    if (chunks <= 512) return forward_as<T, 256, 2>(a, s);
    if (chunks <= 1024) return forward_as<T, 512, 2>(a, s);
    if (chunks <= 2048) return forward_as<T, 1024, 2>(a, s);
    if (chunks <= 4096) return forward_as<T, 1024, 4>(a, s);
    k_norm_forward_wide<T><<<dim3((unsigned)a.rows), 1024, 0, s>>>(a);
    return hipGetLastError();
}
hipError_t launch_norm_forward(const NormForwardLaunch& a, hipStream_t s)
{
    if (a.rows == 0) return hipSuccess;
    return a.dtype == FF_F32 ? forward_of<float>(a, s) : a.dtype == FF_BF16 ? forward_of<bf16_t>(a, s) : forward_of<f16_t>(a, s);
}

// Lanes of a row and workgroups of the backward pass: as many as run at once, each with a share of the rows and one set of column sums.  Up to 1024
// columns a wavefront has a row to itself (131072 x 784 bf16: 237 us by 256 lanes with a chunk each, 144 by 64 with two); up to 1536,
// with three chunks, where there are many (65536 x 1100 bf16: 157 us by 256 lanes, 107 by 64; 2048 rows: 12.2 and 13.6); else up to 2048, 256 lanes with
// one chunk (32768 x 2000 fp32: 147 us, 161 by 128 lanes with two; 2048 x 2000 bf16: 15 and 18).
struct NormPlan {
    int lanes, ch;   // ch == 0: rows too wide for registers
    int64_t wgs;     // workgroups that leave column sums
};
static NormPlan backward_plan(int64_t rows, int64_t cols)
{
    const int64_t chunks = (cols + 7) / 8;
    NormPlan p;
    if (chunks <= 128 || (chunks <= 192 && rows >= 8192)) {
        p.ch = chunks <= 64 ? 1 : chunks <= 128 ? 2 : 3;
        for (p.lanes = 4; p.lanes * p.ch < chunks; p.lanes *= 2) {}
    } else {
        p.lanes = chunks <= 512 ? 256 : 512;
        p.ch = chunks <= 256 ? 1 : chunks <= 1024 ? 2 : chunks <= 2048 ? 4 : 0;
    }
    const int64_t per = p.lanes <= 64 ? 256 / p.lanes : 1;
    const int64_t most = p.ch == 0 ? 64 : p.lanes == 512 ? 256 : p.lanes <= 64 && p.ch < 3 ? 1024 : 512;   // (of 512 lanes a compute unit holds one)
    const int64_t need = (rows + per - 1) / per;
    p.wgs = need < most ? need : most;
    return p;
}
// One launch for rows and columns, or the workgroups' sums and a launch that adds them.  One launch takes time by the rows that a column's workgroup reads, and
// more where rows end inside a chunk, whose loads are behind branches; two are 6 to 20 us nearly whatever the rows.  us, one launch and two, on both sides of the lines:
//   whole chunks        512 x 256 fp32 5.3 and 5.6, 640 x 256 6.0 and 5.9; 768 x 784 fp32 7.5 and 8.1, 768 x 12000 34 and 33, 768 x 16384 45 and 41,
//                       1024 x 784 9.8 and 8.8;
//     up to 16 KB       1024 x 2000 bf16 10.5 and 12.9, 1024 x 4096 fp32 17 and 18, 1024 x 8192 bf16 17.4 and 18.2; beyond: 1024 x 6000 fp32 24 and 21
//   ragged, from x      256 x 783 fp32 7.2 and 7.6, 320 x 783 8.7 and 8.0; 448 x 2001 fp32 11.6 and 12.7, 512 x 2001 14.4 and 13.3, 1024 x 2001 33 and 15; bf16
//                       512 x 2001 11.5 and 13.8, 640 x 3001 19 and 16
//   ragged, from codes  384 x 500 fp32 6.1 and 6.3, 448 x 500 6.6 and 6.4; 384 x 783 7.1 and 7.6, 512 x 783 8.5 and 7.8; 640 x 2001 fp32 11.8 and 14.0, 768 x 2001 14.5 and 14.1; bf16 768 x 2001 10.9 and 13.5,
//                       1024 x 2001 13.6 and 13.2
static bool sums_at_once(const NormPlan& p, int64_t rows, int64_t cols, int size, bool kept)
{
    if (p.ch == 0 || rows == 0) return false;
    if (cols % 8 == 0) return rows <= 512 || (rows <= 768 && cols > 512 && cols * size <= 49152) || (rows <= 1024 && cols > 1024 && cols * size <= 16384);
    if (cols <= 1024) return rows <= (kept ? (cols > 512 ? 448 : 384) : 256);
    return rows <= (kept ? (size == 2 ? 768 : 640) : (size == 2 ? 512 : 448));
}
static int64_t padded_cols(int64_t cols) { return (cols + 7) / 8 * 8; }
size_t norm_backward_workspace(int64_t rows, int64_t cols)
{
    const NormPlan p = backward_plan(rows, cols);
    size_t n = align_up((size_t)(p.wgs * 2 * padded_cols(cols)) * sizeof(float), 256);
    if (p.ch == 0) n += align_up((size_t)rows * sizeof(float2), 256);
    return n < FF_WS_MIN_BYTES ? FF_WS_MIN_BYTES : n;
}

template <typename T, bool KEPT, bool RAGGED> static void backward_by(const NormPlan& p, const NormBackwardArgs<T>& a, int64_t column_wgs, hipStream_t s)
{
    const dim3 grid((unsigned)(a.row_wgs + column_wgs));
    if (p.lanes == 4) k_norm_backward<T, KEPT, 4, 1, RAGGED><<<grid, 256, 0, s>>>(a);
    else if (p.lanes == 8) k_norm_backward<T, KEPT, 8, 1, RAGGED><<<grid, 256, 0, s>>>(a);
    else if (p.lanes == 16) k_norm_backward<T, KEPT, 16, 1, RAGGED><<<grid, 256, 0, s>>>(a);
    else if (p.lanes == 32) k_norm_backward<T, KEPT, 32, 1, RAGGED><<<grid, 256, 0, s>>>(a);
    else if (p.lanes == 64 && p.ch == 1) k_norm_backward<T, KEPT, 64, 1, RAGGED><<<grid, 256, 0, s>>>(a);
    else if (p.lanes == 64 && p.ch == 2) k_norm_backward<T, KEPT, 64, 2, RAGGED><<<grid, 256, 0, s>>>(a);
    else if (p.lanes == 64) k_norm_backward<T, KEPT, 64, 3, RAGGED><<<grid, 256, 0, s>>>(a);
    else if (p.ch == 1) k_norm_backward<T, KEPT, 256, 1, RAGGED><<<grid, 256, 0, s>>>(a);
    else if (p.lanes == 256) k_norm_backward<T, KEPT, 256, 2, RAGGED><<<grid, 256, 0, s>>>(a);
    else if (p.ch == 2) k_norm_backward<T, KEPT, 512, 2, RAGGED><<<grid, 512, 0, s>>>(a);
    else k_norm_backward<T, KEPT, 512, 4, RAGGED><<<grid, 512, 0, s>>>(a);
}
template <typename T, bool KEPT> static hipError_t backward_as(const NormPlan& p, const NormBackwardArgs<T>& a, int64_t column_wgs, hipStream_t s)
{
    if (a.cols % 8 == 0) backward_by<T, KEPT, false>(p, a, column_wgs, s);
    else backward_by<T, KEPT, true>(p, a, column_wgs, s);
    return hipGetLastError();
}
template <typename T, bool KEPT> static hipError_t backward_of(const NormBackwardLaunch& l, hipStream_t s)
{
    const NormPlan p = backward_plan(l.rows, l.cols);
    NormBackwardArgs<T> a;
    a.dy = (const T*)l.dy;
    a.x = (const T*)l.x;
    a.dx = (T*)l.dx;
    a.lddy = l.lddy;
    a.ldx = l.ldx;
    a.lddx = l.lddx;
    a.rows = l.rows;
    a.mean = l.mean;
    a.rstd = l.rstd;
    a.weight = l.weight;
    a.cols = (int32_t)l.cols;
    a.param_f32 = l.param_dtype == FF_F32;
    a.sums = l.dweight || l.dbias;
    a.inv_cols = 1.0f / (float)l.cols;
    a.k = ckpt_ptr(l.q, l.e, l.cols);
    a.part = (float*)l.ws;
    a.pcols = padded_cols(l.cols);
    a.row_sums = (float2*)((char*)l.ws + align_up((size_t)(p.wgs * 2 * a.pcols) * sizeof(float), 256));
    a.dweight = l.dweight;
    a.dbias = l.dbias;
    a.accumulate = l.accumulate;
    const bool at_once = a.sums && sums_at_once(p, l.rows, l.cols, sizeof(T), KEPT);
    const bool in_place = l.dx && (l.dx == l.dy || l.dx == l.x);
    int64_t column_wgs = at_once ? (l.cols + 63) / 64 : 0;
    if (at_once) a.sums = 0;
    if (at_once && (in_place || !l.dx)) {   // the columns alone; in place they are read before any row is written, and added in the same order as elsewhere
        a.row_wgs = 0;
        const hipError_t err = backward_as<T, KEPT>(p, a, column_wgs, s);
        if (err != hipSuccess || !l.dx) return err;
        column_wgs = 0;
    }
    a.row_wgs = p.wgs;
    if (l.rows > 0) {
        if (p.ch == 0) {
            if (a.dx) k_norm_row_sums<T, KEPT><<<dim3((unsigned)l.rows), 1024, 0, s>>>(a);
            k_norm_backward_wide<T, KEPT><<<dim3((unsigned)((a.cols + 2047) / 2048), (unsigned)p.wgs), 256, 0, s>>>(a);
        }
        const hipError_t err = p.ch == 0 ? hipGetLastError() : backward_as<T, KEPT>(p, a, column_wgs, s);
        if (err != hipSuccess) return err;
    }
    if (a.sums) {
        k_norm_columns<<<dim3((unsigned)((a.cols + 31) / 32), 2), 512, 0, s>>>(a.part, l.rows > 0 ? (int)p.wgs : 0, a.pcols, a.cols, l.dweight,
                                                                                l.dbias, l.accumulate);
        return hipGetLastError();
    }
    return hipSuccess;
}
hipError_t launch_norm_backward(const NormBackwardLaunch& a, hipStream_t s)
{
    if (a.dtype == FF_F32) return a.x ? backward_of<float, false>(a, s) : backward_of<float, true>(a, s);
    if (a.dtype == FF_BF16) return a.x ? backward_of<bf16_t, false>(a, s) : backward_of<bf16_t, true>(a, s);
    return a.x ? backward_of<f16_t, false>(a, s) : backward_of<f16_t, true>(a, s);
}

}  // namespace ffi
