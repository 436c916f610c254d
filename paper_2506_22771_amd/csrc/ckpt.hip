// 8-bit checkpoints of activations: written, read back, and read by the gradient through an activation function.
//
//   store:         q, e = codes and exponent bytes of x (ckpt.hpp)            load:  x = q 2^(e - 127)
//   act backward:  dx = (dy + 2 c[row] f(u)) f'(u), u the checkpointed argument of f; 2 c f(u) is the gradient of c G, the goodness
//                  G = sum f(u)^2 of Section III (dL/dG = c), dy what comes down from the layers above (either may be absent)
//
// Measured, us and TB/s, 16384 x 4096, inputs from memory (a copy of as many bytes reaches 5.3): bf16 store 41 (4.9), with stochastic rounding 53 (3.8, by its
// arithmetic: 25 operations a value), load 38 (5.3), ReLU backward 59 (5.7), GELU 64 (5.3); fp32 60 (5.6), 63 (5.3), 69 (4.9), 108 (5.6), 114 (5.3).
// All three are bound by memory but for that.  A lane has eight columns (a chunk) of a row, a quad of lanes one block; a workgroup takes consecutive chunks,
// whatever the row length, and has all its loads in flight before the first is used.
#include "act.hpp"
#include "chunks.hpp"
#include "norm.hpp"

namespace ffi {

template <typename T> struct CkptArgs {
    Chunks c;
    CkptPtr k;
    CkptRound r;
    const T* in;       // store: x; act backward: dy (may be null)
    T* out;            // load: x; act backward: dx
    int64_t ld_in, ld_out;
    const float* coeff;   // act backward: may be null
    int32_t cols, act;
};

template <typename T, RowEnds ENDS, int U> __global__ __launch_bounds__(CK_THREADS) void k_ckpt_store(CkptArgs<T> a)
{
    const int64_t first = (int64_t)blockIdx.x * (CK_THREADS * U);
    int64_t row0;
    uint32_t chunk0;
    chunk_first(a.c, first, row0, chunk0);
    Raw8<T> raw[U];
    uint32_t r[U], chunk[U];
    int n[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        n[i] = chunk_at(a.c, a.cols, first, chunk0, i * CK_THREADS + threadIdx.x, r[i], chunk[i]);
        raw[i] = row_chunk<ENDS>(element(a.in, a.ld_in, row0, r[i], 0), (int)chunk[i], n[i], a.cols);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        float v[8];
        settle<ENDS>(raw[i], n[i], a.cols);
        raw_values(raw[i], v);
        const uint32_t m = quad_max_u32(abs_max_bits(v)), e = ckpt_exponent(m);
        const u32x2 q = ckpt_codes(v, m, e, a.r, (uint64_t)row0 * (uint64_t)a.cols + ((uint64_t)r[i] * (uint32_t)a.cols + 8 * chunk[i]));
        if (first + i * CK_THREADS + threadIdx.x < a.c.total)
            ckpt_store_chunk(a.k, element(a.k.q, a.k.pitch, row0, r[i], 0), element(a.k.e, a.k.epitch, row0, r[i], 0), (int)chunk[i], (int)a.c.slots,
                             n[i] > 0, q, e);
    }
}

// A code rounded up can stand for more than fp16 holds (65504 becomes 64 * 2^10): given as the largest value.
template <typename T> __device__ __forceinline__ float ckpt_clamp(float v) { return v; }
template <> __device__ __forceinline__ float ckpt_clamp<f16_t>(float v) { return v == v ? __builtin_amdgcn_fmed3f(v, -65504.0f, 65504.0f) : v; }

// (Its loads are behind branches, one chunk's after the other's: all at once, 16384 x 4096 fp32 values took 80 us in the place of 71.)
template <typename T, int U> __global__ __launch_bounds__(CK_THREADS) void k_ckpt_load(CkptArgs<T> a)
{
    const int64_t first = (int64_t)blockIdx.x * (CK_THREADS * U);
    int64_t row0;
    uint32_t chunk0;
    chunk_first(a.c, first, row0, chunk0);
    u32x2 q[U];
    uint32_t e[U];
    T* to[U];
    int n[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        uint32_t r, chunk;
        n[i] = chunk_at(a.c, a.cols, first, chunk0, i * CK_THREADS + threadIdx.x, r, chunk);
        to[i] = element(a.out, a.ld_out, row0, r, 8 * chunk);
        q[i] = u32x2{0, 0};
        e[i] = 127;
        if (n[i] > 0) {
            q[i] = *(const u32x2*)element(a.k.q, a.k.pitch, row0, r, 8 * chunk);
            e[i] = *element(a.k.e, a.k.epitch, row0, r, chunk >> 2);
        }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        float v[8];
        ckpt_values(q[i], e[i], v);
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = ckpt_clamp<T>(v[u]);
        if (n[i] > 0) store8(to[i], n[i], v);
    }
}

template <typename T, int ACT, RowEnds ENDS, int U> __global__ __launch_bounds__(CK_THREADS) void k_ckpt_act_backward(CkptArgs<T> a)
{
    const int64_t first = (int64_t)blockIdx.x * (CK_THREADS * U);
    int64_t row0;
    uint32_t chunk0;
    chunk_first(a.c, first, row0, chunk0);
    // dy or c that is not there is zero: its loads all go to one place that is there, and count for nothing
    const T* const in = a.in ? a.in : a.out;
    const int64_t ld_in = a.in ? a.ld_in : 0, ld_c = a.coeff ? 1 : 0;
    const float* const coeff = a.coeff ? a.coeff : (const float*)a.k.q;
    const uint32_t c_mask = a.coeff ? 0xFFFFFFFFu : 0u;
    Raw8<T> raw[U];
    u32x2 q[U];
    uint32_t e[U];
    float c[U];
    T* to[U];
    int n[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        uint32_t r, chunk;
        n[i] = chunk_at(a.c, a.cols, first, chunk0, i * CK_THREADS + threadIdx.x, r, chunk);
        to[i] = element(a.out, a.ld_out, row0, r, 8 * chunk);
        raw[i] = row_chunk<ENDS>(element(in, ld_in, row0, r, 0), (int)chunk, a.in ? n[i] : 0, a.cols);
        chunk = n[i] > 0 ? chunk : 0;   // (the row's pitch ends before its last block)
        q[i] = *(const u32x2*)element(a.k.q, a.k.pitch, row0, r, 8 * chunk);
        e[i] = *element(a.k.e, a.k.epitch, row0, r, chunk >> 2);
        c[i] = *element(coeff, ld_c, row0, r, 0);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        float u[8], v[8];
        settle<ENDS>(raw[i], a.in ? n[i] : 0, a.cols);
        const float c2 = 2.0f * __uint_as_float(__float_as_uint(c[i]) & c_mask);
        ckpt_values(q[i], e[i], u);
        raw_values(raw[i], v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float f, d;
            act_of<T, ACT>(u[j], f, d);
            // (c2 = 0 where there is no c: f is finite, or it is NaN and so is d, but for the identity's)
            v[j] = ACT == FF_ACT_IDENTITY && !a.coeff ? v[j] : __builtin_fmaf(c2, f, v[j]) * d;
        }
        if (n[i] > 0) store8(to[i], n[i], v);
    }
}

// ------------------------------------------------------------------------------------------------
// launches
// ------------------------------------------------------------------------------------------------
template <typename T> static CkptArgs<T> ckpt_args(const int8_t* q, const uint8_t* e, int64_t rows, int64_t cols, int64_t span)
{
    CkptArgs<T> a = {};
    a.c = chunks_of(rows, span);
    a.k = ckpt_ptr(q, e, cols);
    a.cols = (int32_t)cols;
    return a;
}
template <typename T> static hipError_t store_of(const void* x, int64_t ldx, int64_t rows, int64_t cols, const CkptRound& r, int8_t* q, uint8_t* e, hipStream_t s)
{
    CkptArgs<T> a = ckpt_args<T>(q, e, rows, cols, pitch8(cols));   // pad columns are written too
    a.in = (const T*)x;
    a.ld_in = ldx;
    a.r = r;
    by_ends(cols, false, [&](auto ends) { k_ckpt_store<T, decltype(ends)::value, 2><<<ckpt_grid<2>(a.c), CK_THREADS, 0, s>>>(a); });
    return hipGetLastError();
}
hipError_t launch_ckpt_store(const void* x, int32_t dtype, int64_t ldx, int64_t rows, int64_t cols, int32_t round_mode, uint64_t seed,
                             uint64_t tag, int8_t* q, uint8_t* e, hipStream_t s)
{
    if (rows == 0) return hipSuccess;
    const CkptRound r = {make_sr_key(seed, tag), round_mode == FF_ROUND_STOCHASTIC};
    return dtype == FF_F32    ? store_of<float>(x, ldx, rows, cols, r, q, e, s)
           : dtype == FF_BF16 ? store_of<bf16_t>(x, ldx, rows, cols, r, q, e, s)
                              : store_of<f16_t>(x, ldx, rows, cols, r, q, e, s);
}

template <typename T> static hipError_t load_of(const int8_t* q, const uint8_t* e, int64_t rows, int64_t cols, void* x, int64_t ldx, hipStream_t s)
{
    CkptArgs<T> a = ckpt_args<T>(q, e, rows, cols, cols);
    a.out = (T*)x;
    a.ld_out = ldx;
    k_ckpt_load<T, 2><<<ckpt_grid<2>(a.c), CK_THREADS, 0, s>>>(a);
    return hipGetLastError();
}
hipError_t launch_ckpt_load(const int8_t* q, const uint8_t* e, int64_t rows, int64_t cols, void* x, int32_t dtype, int64_t ldx,
                            hipStream_t s)
{
    if (rows == 0) return hipSuccess;
    return dtype == FF_F32    ? load_of<float>(q, e, rows, cols, x, ldx, s)
           : dtype == FF_BF16 ? load_of<bf16_t>(q, e, rows, cols, x, ldx, s)
                              : load_of<f16_t>(q, e, rows, cols, x, ldx, s);
}

template <typename T>
static hipError_t act_backward_of(const int8_t* q, const uint8_t* e, int64_t rows, int64_t cols, int32_t act, const float* coeff, const void* dy,
                                  int64_t lddy, void* dx, int64_t lddx, hipStream_t s)
{
    CkptArgs<T> a = ckpt_args<T>(q, e, rows, cols, cols);
    a.in = (const T*)dy;
    a.ld_in = lddy;
    a.out = (T*)dx;
    a.ld_out = lddx;
    a.coeff = coeff;
    const unsigned grid = ckpt_grid<2>(a.c);
    by_ends(cols, dy == dx, [&](auto ends) {
        constexpr RowEnds E = decltype(ends)::value;
        switch (act) {
            case FF_ACT_RELU: k_ckpt_act_backward<T, FF_ACT_RELU, E, 2><<<grid, CK_THREADS, 0, s>>>(a); break;
            case FF_ACT_GELU: k_ckpt_act_backward<T, FF_ACT_GELU, E, 2><<<grid, CK_THREADS, 0, s>>>(a); break;
            case FF_ACT_SILU: k_ckpt_act_backward<T, FF_ACT_SILU, E, 2><<<grid, CK_THREADS, 0, s>>>(a); break;
            default: k_ckpt_act_backward<T, FF_ACT_IDENTITY, E, 2><<<grid, CK_THREADS, 0, s>>>(a); break;
        }
    });
    return hipGetLastError();
}
hipError_t launch_ckpt_act_backward(const int8_t* q, const uint8_t* e, int64_t rows, int64_t cols, int32_t act, const float* coeff,
                                    const void* dy, int64_t lddy, void* dx, int64_t lddx, int32_t dtype, hipStream_t s)
{
    if (rows == 0) return hipSuccess;
    return dtype == FF_F32    ? act_backward_of<float>(q, e, rows, cols, act, coeff, dy, lddy, dx, lddx, s)
           : dtype == FF_BF16 ? act_backward_of<bf16_t>(q, e, rows, cols, act, coeff, dy, lddy, dx, lddx, s)
                              : act_backward_of<f16_t>(q, e, rows, cols, act, coeff, dy, lddy, dx, lddx, s);
}

}  // namespace ffi
