// A gated layer's forward pass: both int8 projections, the activation, the product, and what training keeps of them, in one kernel.
//
//   s = s_a s_w,   g = s a_q Wg_q^T,   u = s a_q Wu_q^T,   y = f(g) u,   G[row] = sum y^2;   optionally the 8-bit checkpoints of g and u
//
// w_q is one int8 matrix [2n, k], the gate's rows first.  A workgroup contracts the same columns of both projections, so that a lane holds g and u of one
// place and neither is ever in memory at more than 8 bits.  Accumulators are exact; g and u are the int32 sums, rounded to fp32, times s.
#include <algorithm>
#include <type_traits>

#include "act.hpp"
#include "blocks.hpp"

namespace ffi {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));

struct GatedArgs {
    const int8_t* a_q;
    const int8_t* w_q;
    const float* s_a;
    const float* s_w;
    int64_t ld;       // row pitch of both
    int32_t rows, n, k, act;
    void* y;
    int64_t ldy;
    CkptPtr g, u;     // q null: nothing is kept
    float* good;      // sums of squares of every 32 or 128 columns, [..][rows]; or null
};

__device__ __forceinline__ float dpp_add8(float v)   // sum over eight consecutive lanes
{
    v += __uint_as_float(dpp_u32<0xB1>(__float_as_uint(v)));
    v += __uint_as_float(dpp_u32<0x4E>(__float_as_uint(v)));
    v += __uint_as_float(dpp_u32<0x141>(__float_as_uint(v)));
    return v;
}
__device__ __forceinline__ uint32_t dpp_max8(uint32_t v)
{
    v = quad_max_u32(v);
    return max(v, dpp_u32<0x141>(v));
}
// f(g) u of four places
template <typename T> __device__ __forceinline__ void gate4(int act, const float g[4], const float u[4], float y[4])
{
    auto of = [&](auto kind) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float f, d;
            act_of<T, decltype(kind)::value, true>(g[i], f, d);
            y[i] = f * u[i];
        }
    };
    switch (act) {   // (uniform)
        case FF_ACT_RELU: of(std::integral_constant<int, FF_ACT_RELU>()); break;
        case FF_ACT_GELU: of(std::integral_constant<int, FF_ACT_GELU>()); break;
        case FF_ACT_SILU: of(std::integral_constant<int, FF_ACT_SILU>()); break;
        default: of(std::integral_constant<int, FF_ACT_IDENTITY>());
    }
}
__device__ __forceinline__ uint32_t abs_max_bits4(const float v[4])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return m;
}
// Codes of four values, rounded to nearest, of a block of this absmax and exponent: ckpt_codes' arithmetic.
__device__ __forceinline__ uint32_t codes4(const float v[4], uint32_t top, uint32_t e)
{
    const bool some = top >= (27u << 23) && top < 0x7F800000u;
    const float inv = __uint_as_float((254u - e) << 23);
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __float_as_uint(__builtin_amdgcn_fmed3f(v[i] * inv, -127.0f, 127.0f) + 12582912.0f);
    const uint32_t lo = __builtin_amdgcn_perm(x[1], x[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(x[3], x[2], 0x04000C0Cu);
    return some ? lo | hi : 0u;
}
// n (1 .. 4) values
__device__ __forceinline__ void store4(float* p, int n, const float v[4])
{
    if (n >= 4) write_as<u32x4>(p, u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
    else
        for (int i = 0; i < 3; ++i)
            if (i < n) p[i] = v[i];
}
__device__ __forceinline__ void store4_words(uint16_t* p, int n, uint32_t a, uint32_t b)
{
    if (n >= 4) write_as<u32x2>(p, u32x2{a, b});
    else {
        p[0] = (uint16_t)a;
        if (n > 1) p[1] = (uint16_t)(a >> 16);
        if (n > 2) p[2] = (uint16_t)b;
    }
}
__device__ __forceinline__ void store4(bf16_t* p, int n, const float v[4]) { store4_words((uint16_t*)p, n, bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])); }
__device__ __forceinline__ void store4(f16_t* p, int n, const float v[4]) { store4_words((uint16_t*)p, n, f16_pair(v[0], v[1]), f16_pair(v[2], v[3])); }

// ------------------------------------------------------------------------------------------------
// Tiles of 32 x 32 outputs: four wavefronts share out the reduction, each with 96 rows of operands (samples, gate, value) of every fourth step of 128 bytes.
// ------------------------------------------------------------------------------------------------
constexpr int WAVES = 4, D = 2;   // wavefronts of a workgroup, steps of each in flight

template <typename T> __global__ __launch_bounds__(WAVES * 64) void k_gated_few(GatedArgs a, int ntiles, int per_xcd)
{
    constexpr int EROW = 36, MINE = 3 * 4096;   // words between rows of partial sums, bytes of a wavefront
    __shared__ __attribute__((aligned(16))) int8_t lds[WAVES * MINE];
    // workgroups go to the eight XCDs in turn: each XCD gets consecutive tiles, which share their columns' weights in its L2
    const int t = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
    if (t >= ntiles) return;
    const int tiles_i = (a.rows + 31) / 32;
    const int bj = t / tiles_i, bi = t - bj * tiles_i;
    const int i0 = bi * 32, j0 = bj * 32;
    const int jrows = min(32, a.n - j0), irows = min(32, a.rows - i0);
    // rows beyond the matrices and bytes beyond the reduction read as zero (range check of the buffer)
    const __amdgpu_buffer_rsrc_t rp = __builtin_amdgcn_make_buffer_rsrc((void*)(a.a_q + (int64_t)i0 * a.ld), 0, (int)(irows * a.ld), 0x00020000);
    const __amdgpu_buffer_rsrc_t rg = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w_q + (int64_t)j0 * a.ld), 0, (int)(jrows * a.ld), 0x00020000);
    const __amdgpu_buffer_rsrc_t ru = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w_q + (int64_t)(a.n + j0) * a.ld), 0, (int)(jrows * a.ld), 0x00020000);
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, lh = lane >> 5, r8 = lane >> 3, ch = lane & 7;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kpad = (a.k + 15) & ~15;
    const int nk = (kpad + 127) >> 7;
    const int n = nk > wave ? (nk - wave + WAVES - 1) / WAVES : 0;   // this wavefront's steps
    const int row8 = r8 * (int)a.ld, by8 = 8 * (int)a.ld;
    int8_t* const mine = lds + wave * MINE;

    v4i p[D][4], g[D][4], u[D][4];
    // load c: rows 8 c .. 8 c + 7, eight lanes to a row's 128 bytes
    auto load = [&](int s, int d) {
        const int k = (wave + s * WAVES) * 128 + ch * 16;
        const bool in = k < kpad;
#pragma unroll
        for (int c = 0; c < 4; ++c) p[d][c] = (v4i)__builtin_amdgcn_raw_buffer_load_b128(rp, in ? row8 + c * by8 + k : 0x7FFFFFF0, 0, 0);
#pragma unroll
        for (int c = 0; c < 4; ++c) g[d][c] = (v4i)__builtin_amdgcn_raw_buffer_load_b128(rg, in ? row8 + c * by8 + k : 0x7FFFFFF0, 0, 0);
#pragma unroll
        for (int c = 0; c < 4; ++c) u[d][c] = (v4i)__builtin_amdgcn_raw_buffer_load_b128(ru, in ? row8 + c * by8 + k : 0x7FFFFFF0, 0, 0);
    };
    v16i ag, au;
#pragma unroll
    for (int e = 0; e < 16; ++e) ag[e] = au[e] = 0;
#pragma unroll
    for (int d = 0; d < D; ++d) load(d, d);
    for (int s = 0; s < n; s += D) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            if (s + d >= n) break;   // (uniform)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int row = 8 * c + r8, at = row * 128 + ((ch ^ ((row >> 1) & 7)) << 4);
                *(v4i*)(mine + at) = p[d][c];
                *(v4i*)(mine + 4096 + at) = g[d][c];
                *(v4i*)(mine + 8192 + at) = u[d][c];
            }
            load(s + d + D, d);
            wave_lds_fence();
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const int at = lr * 128 + (((2 * m + lh) ^ ((lr >> 1) & 7)) << 4);
                const v4i fp = *(const v4i*)(mine + at), fg = *(const v4i*)(mine + 4096 + at), fu = *(const v4i*)(mine + 8192 + at);
                ag = __builtin_amdgcn_mfma_i32_32x32x32_i8(fg, fp, ag, 0, 0, 0);
                au = __builtin_amdgcn_mfma_i32_32x32x32_i8(fu, fp, au, 0, 0, 0);
            }
            wave_lds_fence();
        }
    }
    // lane: row lr, columns 8 q + 4 lh .. + 3
    wave_lds_fence();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        *(v4i*)(mine + (lr * EROW + 8 * q + 4 * lh) * 4) = (v4i){ag[4 * q + 0], ag[4 * q + 1], ag[4 * q + 2], ag[4 * q + 3]};
        *(v4i*)(mine + (32 * EROW + lr * EROW + 8 * q + 4 * lh) * 4) = (v4i){au[4 * q + 0], au[4 * q + 1], au[4 * q + 2], au[4 * q + 3]};
    }
    __syncthreads();
    // eight lanes to a row, four columns each
    const int row = tid >> 3, cc = (tid & 7) * 4, i = i0 + row, j = j0 + cc;
    v4i vg = {0, 0, 0, 0}, vu = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        vg += *(const v4i*)(lds + w * MINE + (row * EROW + cc) * 4);
        vu += *(const v4i*)(lds + w * MINE + (32 * EROW + row * EROW + cc) * 4);
    }
    const float sc = a.s_a[0] * a.s_w[0];
    float fg[4], fu[4], y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        fg[e] = (float)vg[e] * sc;
        fu[e] = (float)vu[e] * sc;
        // columns beyond the matrix are no part of a block (their sums are zero, but the scale may be anything)
        if (j + e >= a.n) fg[e] = fu[e] = 0.0f;
    }
    gate4<T>(a.act, fg, fu, y);
    if (i < a.rows && j < a.n) store4((T*)a.y + ((int64_t)i * a.ldy + j), a.n - j, y);
    if (a.good) {
        float s = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) s = j + e < a.n ? __builtin_fmaf(y[e], y[e], s) : s;
        s = dpp_add8(s);
        if ((tid & 7) == 0 && i < a.rows) a.good[(int64_t)bj * a.rows + i] = s;
    }
    if (a.g.q) {   // a row's 32 columns are a block
        const bool last = j0 + 32 >= a.n;
        auto keep = [&](const CkptPtr& k, const float v[4]) {
            const uint32_t top = dpp_max8(abs_max_bits4(v)), e = ckpt_exponent(top), q = codes4(v, top, e);
            if (i >= a.rows) return;
            int8_t* const qr = k.q + (int64_t)i * k.pitch;
            uint8_t* const er = k.e + (int64_t)i * k.epitch;
            if (j < k.pitch) *(uint32_t*)(qr + j) = q;
            if ((tid & 7) == 0) er[bj] = (uint8_t)e;
            if (last) {   // the pads
                for (int64_t at = j + 32; at < k.pitch; at += 32) *(uint32_t*)(qr + at) = 0;
                for (int at = k.blocks + (tid & 7); at < (int)k.epitch; at += 8) er[at] = 0;
            }
        };
        keep(a.g, fg);
        keep(a.u, fu);
    }
}

// goodness[row] = its parts in their order
__global__ __launch_bounds__(256) void k_gated_goodness(const float* part, float* goodness, int32_t rows, int32_t parts)
{
    const int row = (int)(blockIdx.x * 256 + threadIdx.x);
    if (row >= rows) return;
    float s = 0;
#pragma unroll 8
    for (int p = 0; p < parts; ++p) s += part[(int64_t)p * rows + row];
    goodness[row] = s;
}

// ------------------------------------------------------------------------------------------------
// launches
// ------------------------------------------------------------------------------------------------
size_t gated_workspace(int64_t rows, int64_t n, int64_t)
{
    return align_up(std::max<size_t>((size_t)(rows * ((n + 31) / 32)) * sizeof(float), FF_WS_MIN_BYTES), 16);
}

template <typename T> static hipError_t forward_of(GatedArgs a, float* goodness, hipStream_t s)
{
    const int64_t parts = (a.n + 31) / 32, ntiles = (int64_t)((a.rows + 31) / 32) * parts;
    const int per_xcd = (int)((ntiles + 7) / 8);
    if (goodness && parts == 1) a.good = goodness;
    k_gated_few<T><<<(unsigned)(8 * per_xcd), WAVES * 64, 0, s>>>(a, (int)ntiles, per_xcd);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (goodness && parts > 1) k_gated_goodness<<<(unsigned)((a.rows + 255) / 256), 256, 0, s>>>(a.good, goodness, a.rows, (int32_t)parts);
    return hipGetLastError();
}
hipError_t launch_gated_forward(const GatedForwardLaunch& f, hipStream_t s)
{
    GatedArgs a = {};
    a.a_q = f.a_q;
    a.w_q = f.w_q;
    a.s_a = f.s_a;
    a.s_w = f.s_w;
    a.ld = pitch8(f.k);
    a.rows = (int32_t)f.rows;
    a.n = (int32_t)f.n;
    a.k = (int32_t)f.k;
    a.act = f.act;
    a.y = f.y;
    a.ldy = f.ldy;
    if (f.qg) {
        a.g = ckpt_ptr(f.qg, f.eg, f.n);
        a.u = ckpt_ptr(f.qu, f.eu, f.n);
    }
    a.good = f.goodness ? (float*)f.ws : nullptr;
    return f.dtype == FF_F32    ? forward_of<float>(a, f.goodness, s)
           : f.dtype == FF_BF16 ? forward_of<bf16_t>(a, f.goodness, s)
                                : forward_of<f16_t>(a, f.goodness, s);
}

}  // namespace ffi
