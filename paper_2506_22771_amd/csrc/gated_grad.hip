// Gradient through a gated layer's activation and product, from the 8-bit checkpoints of both projections:
//
//   t = dy + 2 c[row] f(g) u,   dg = t u f'(g),   du = t f(g)
//
// The second term of t is the gradient of c G, G = sum (f(g) u)^2 the goodness of the row.  Bound by memory: two codes and dy are read, two values written.
// Measured: 16384 x 4096 bf16 SiLU with both terms 93 us (5.8 TB/s, 27 vector instructions a value); 128 x 500 fp32 GELU 6.6 us a call.
#include "act.hpp"
#include "blocks.hpp"
#include "chunks.hpp"

namespace ffi {

template <typename T> struct GatedGradArgs {
    Chunks c;
    CkptPtr g, u;
    const T* dy;          // may be null
    const float* coeff;   // may be null
    T* dg;
    T* du;
    int64_t lddy, lddg, lddu;
    int32_t cols;
};

template <typename T, int ACT, RowEnds ENDS, int U> __global__ __launch_bounds__(CK_THREADS) void k_gated_grad(GatedGradArgs<T> a)
{
    const int64_t first = (int64_t)blockIdx.x * (CK_THREADS * U);
    int64_t row0;
    uint32_t chunk0;
    chunk_first(a.c, first, row0, chunk0);
    // dy or c that is not there is zero: its loads all go to one place that is there, and count for nothing
    const T* const in = a.dy ? a.dy : a.dg;
    const int64_t ld_in = a.dy ? a.lddy : 0, ld_c = a.coeff ? 1 : 0;
    const float* const coeff = a.coeff ? a.coeff : (const float*)a.g.q;
    const uint32_t c_mask = a.coeff ? 0xFFFFFFFFu : 0u;
    Raw8<T> raw[U];
    u32x2 qg[U], qu[U];
    uint32_t eg[U], eu[U], r[U], chunk[U];
    float c[U];
    int n[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        n[i] = chunk_at(a.c, a.cols, first, chunk0, i * CK_THREADS + threadIdx.x, r[i], chunk[i]);
        raw[i] = row_chunk<ENDS>(element(in, ld_in, row0, r[i], 0), (int)chunk[i], a.dy ? n[i] : 0, a.cols);
        const uint32_t at = n[i] > 0 ? chunk[i] : 0;   // (the row's pitch ends before its last block)
        qg[i] = *(const u32x2*)element(a.g.q, a.g.pitch, row0, r[i], 8 * at);
        eg[i] = *element(a.g.e, a.g.epitch, row0, r[i], at >> 2);
        qu[i] = *(const u32x2*)element(a.u.q, a.u.pitch, row0, r[i], 8 * at);
        eu[i] = *element(a.u.e, a.u.epitch, row0, r[i], at >> 2);
        c[i] = *element(coeff, ld_c, row0, r[i], 0);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        float g[8], u[8], t[8];
        settle<ENDS>(raw[i], a.dy ? n[i] : 0, a.cols);
        const float c2 = 2.0f * __uint_as_float(__float_as_uint(c[i]) & c_mask);
        ckpt_values(qg[i], eg[i], g);
        ckpt_values(qu[i], eu[i], u);
        raw_values(raw[i], t);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float f, d;
            act_of<T, ACT, true>(g[j], f, d);
            if (a.coeff) t[j] = __builtin_fmaf(c2, f * u[j], t[j]);   // (uniform)
            g[j] = t[j] * u[j] * d;
            u[j] = t[j] * f;
        }
        if (n[i] > 0) {
            store8(element(a.dg, a.lddg, row0, r[i], 8 * chunk[i]), n[i], g);
            store8(element(a.du, a.lddu, row0, r[i], 8 * chunk[i]), n[i], u);
        }
    }
}

template <typename T> static hipError_t grad_of(const GatedBackwardLaunch& b, hipStream_t s)
{
    GatedGradArgs<T> a = {};
    a.c = chunks_of(b.rows, b.n);
    a.g = ckpt_ptr(b.qg, b.eg, b.n);
    a.u = ckpt_ptr(b.qu, b.eu, b.n);
    a.dy = (const T*)b.dy;
    a.coeff = b.coeff;
    a.dg = (T*)b.dg;
    a.du = (T*)b.du;
    a.lddy = b.lddy;
    a.lddg = b.lddg;
    a.lddu = b.lddu;
    a.cols = (int32_t)b.n;
    const unsigned grid = ckpt_grid<2>(a.c);
    by_ends(b.n, b.dy == b.dg || b.dy == b.du, [&](auto ends) {
        constexpr RowEnds E = decltype(ends)::value;
        switch (b.act) {
            case FF_ACT_RELU: k_gated_grad<T, FF_ACT_RELU, E, 2><<<grid, CK_THREADS, 0, s>>>(a); break;
            case FF_ACT_GELU: k_gated_grad<T, FF_ACT_GELU, E, 2><<<grid, CK_THREADS, 0, s>>>(a); break;
            case FF_ACT_SILU: k_gated_grad<T, FF_ACT_SILU, E, 2><<<grid, CK_THREADS, 0, s>>>(a); break;
            default: k_gated_grad<T, FF_ACT_IDENTITY, E, 2><<<grid, CK_THREADS, 0, s>>>(a); break;
        }
    });
    return hipGetLastError();
}
hipError_t launch_gated_backward(const GatedBackwardLaunch& b, hipStream_t s)
{
    return b.dtype == FF_F32 ? grad_of<float>(b, s) : b.dtype == FF_BF16 ? grad_of<bf16_t>(b, s) : grad_of<f16_t>(b, s);
}

}  // namespace ffi
