// A gated layer's forward pass: both int8 projections, the activation, the product, and what training keeps of them, in one kernel.
//
//   s = s_a s_w,   g = s a_q Wg_q^T,   u = s a_q Wu_q^T,   y = f(g) u,   G[row] = sum y^2;   optionally the 8-bit checkpoints of g and u
//
// w_q is one int8 matrix [2n, k], the gate's rows first.  A workgroup contracts the same columns of both projections, so that a lane holds g and u of one
// place and neither is ever in memory at more than 8 bits.  Accumulators are exact; g and u are the int32 sums, rounded to fp32, times s.
#include <algorithm>
#include <type_traits>
#include <utility>

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
// f(g) u of N places
template <typename T, int N> __device__ __forceinline__ void gate(int act, const float (&g)[N], const float (&u)[N], float (&y)[N])
{
    auto of = [&](auto kind) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
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
// four values at an aligned place in LDS
__device__ __forceinline__ void stage4(float* p, const float v[4]) { *(u32x4*)p = u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}; }
__device__ __forceinline__ void stage4(bf16_t* p, const float v[4]) { *(u32x2*)p = u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])}; }
__device__ __forceinline__ void stage4(f16_t* p, const float v[4]) { *(u32x2*)p = u32x2{f16_pair(v[0], v[1]), f16_pair(v[2], v[3])}; }
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
    gate<T>(a.act, fg, fu, y);
    if (i < a.rows && j < a.n) store4((T*)a.y + ((int64_t)i * a.ldy + j), a.n - j, y);
    if (a.good) {
        float s = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_fmaf(y[e], y[e], s);   // (zero beyond the matrix)
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

// ------------------------------------------------------------------------------------------------
// Tiles of BM rows x BN outputs (2 BN rows of weights) for many rows: the contraction's pipeline (gemm_i8.hip) over three operands.  Steps of 128 bytes of the
// reduction go from memory straight into two LDS stages; 16-byte chunks are swizzled inside their rows; fragments are double-buffered in registers; half of the
// wavefronts issue a step's copies before its last multiplies and half after them.  A wavefront has the same 32 columns of both projections, which is one
// checkpoint block: its exponent takes a maximum inside a lane and one exchange.  A workgroup takes tile after tile, the next one's first copies under way
// during the epilogue; tiles go to an XCD in blocks of eight rows of tiles, which share operands in its L2.
// 16384 x 4096 x 4096 bf16, kept: 504 to 525 us, 1.10e12 operations at 2.1 to 2.2 POP/s (602 to 606 where the clock falls under the load: box by box, and under a profiler), where a library's int8 product alone takes 558.  The matrix pipe is busy for half of
// the clocks (beside it, LDS reads take 384 of every 512: six fragments to eight multiplies), and 280 MB of stores are 50 us.  Short reductions are bound by the epilogue:
// 16384 x 64 x 1024 bf16, kept, 26 us, 68 MB written; 60000 x 128 x 1000 fp32 69 us, 240 MB.
// ------------------------------------------------------------------------------------------------
template <int N> __device__ __forceinline__ void wait_copies()   // all but N of this wavefront's copies and stores
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// 16 bytes a lane from a buffer straight into LDS at lds_base + AT + lane * 16; completion is tracked by hand.  (The sum is made where it is used: kept, those of both
// stages are more scalars than there are.)
template <int AT> __device__ __forceinline__ void copy16(__amdgpu_buffer_rsrc_t rsrc, int voffset, int soffset, unsigned lds_base)
{
    asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds_base), "v"(voffset), "s"(rsrc), "s"(soffset), "n"(AT) : "memory", "m0", "scc");
}
// each(0), ..., each(N - 1), as constants
template <typename F, int... I> __device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F&& each) { (each(std::integral_constant<int, I>()), ...); }
constexpr int BEYOND = 0x7FFFFFF0;   // a byte offset beyond any buffer
__device__ __forceinline__ int swizzled(int row, int chunk) { return row * 128 + ((chunk ^ ((row >> 1) & 7)) << 4); }

struct GatedTiles {
    int32_t i, j, all, per_turn;   // tiles of rows, of columns, in all; workgroups of an XCD
};
// Tile t of the order: blocks of eight rows of tiles, columns after columns.
__device__ __forceinline__ void tile_of(const GatedTiles& t, int at, int& bi, int& bj)
{
    const int block = at / (8 * t.j), first = block * 8, high = min(8, t.i - first), rest = at - first * t.j;
    bj = rest / high;
    bi = first + (rest - bj * high);
}

// Bits of the largest magnitude of a lane's and its partner's (32 lanes on) sums, scaled.
__device__ __forceinline__ uint32_t abs_max16(const v16i& sum, float scale)
{
    int hi = sum[0], lo = sum[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) {
        hi = max(hi, sum[e]);
        lo = min(lo, sum[e]);
    }
    const int m = max(hi, -lo);   // (sums are below 2^31)
    return __float_as_uint((float)max(m, __shfl_xor(m, 32)) * scale) & 0x7FFFFFFFu;
}

template <typename T, int BM, int BN, int WM, int WN> __global__ __launch_bounds__(WM* WN * 64) void k_gated_tiles(GatedArgs a, GatedTiles tiles)
{
    constexpr int THREADS = WM * WN * 64, TI = BM / WM / 32;
    constexpr int CH_P = BM * 8 / THREADS, CH_W = BN * 8 / THREADS, CH = CH_P + 2 * CH_W;   // copies of a thread per step
    constexpr int STAGE = (BM + 2 * BN) * 128;
    static_assert(BN == 32 * WN && BM * 8 % THREADS == 0 && BN * 8 % THREADS == 0 && THREADS / 8 % 16 == 0, "tile and threads");
    // a wavefront's staging: 32 rows of y, of g's codes and of u's, each padded
    constexpr int YROW = 32 * (int)sizeof(T) + 16, QROW = 48, STAGED = 32 * (YROW + 2 * QROW);
    static_assert(STAGED * WM * WN <= STAGE, "staging");
    __shared__ __attribute__((aligned(16))) int8_t lds[2 * STAGE];
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
    const int kpad = (a.k + 15) & ~15, nk = (kpad + 127) >> 7;
    const int kcol = ((tid & 7) ^ (((tid >> 3) >> 1) & 7)) * 16;
    const float sc = a.s_a[0] * a.s_w[0];
    int off_p[CH_P], off_w[CH_W];
#pragma unroll
    for (int s = 0; s < CH_P; ++s) off_p[s] = ((s * THREADS + tid) >> 3) * (int)a.ld + kcol;
#pragma unroll
    for (int s = 0; s < CH_W; ++s) off_w[s] = ((s * THREADS + tid) >> 3) * (int)a.ld + kcol;
    __amdgpu_buffer_rsrc_t rp, rg, ru;
    auto operands = [&](int bi, int bj) {
        const int irows = min(BM, a.rows - bi * BM), jrows = min(BN, a.n - bj * BN);
        rp = __builtin_amdgcn_make_buffer_rsrc((void*)(a.a_q + (int64_t)bi * BM * a.ld), 0, (int)(irows * a.ld), 0x00020000);
        rg = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w_q + (int64_t)bj * BN * a.ld), 0, (int)(jrows * a.ld), 0x00020000);
        ru = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w_q + (int64_t)(a.n + bj * BN) * a.ld), 0, (int)(jrows * a.ld), 0x00020000);
    };
    auto issue = [&](int kt, int buf) {
        const int k0 = __builtin_amdgcn_readfirstlane(kt * 128);
        const bool in = k0 + kcol < kpad;   // only the last step has chunks beyond the reduction
        const unsigned base = (unsigned)(uintptr_t)(lds + buf * STAGE + wave * 1024);
        each_of(std::make_integer_sequence<int, CH_P>(), [&](auto s) { copy16<s * THREADS * 16>(rp, in ? off_p[s] : BEYOND - k0, k0, base); });
        each_of(std::make_integer_sequence<int, CH_W>(), [&](auto s) { copy16<BM * 128 + s * THREADS * 16>(rg, in ? off_w[s] : BEYOND - k0, k0, base); });
        each_of(std::make_integer_sequence<int, CH_W>(), [&](auto s) { copy16<(BM + BN) * 128 + s * THREADS * 16>(ru, in ? off_w[s] : BEYOND - k0, k0, base); });
    };
    const bool early = wave < WM * WN / 2;
    bool prefetched = false;
    for (int turn = (int)(blockIdx.x & 7) * tiles.per_turn + (int)(blockIdx.x >> 3); turn < tiles.all; turn += (int)gridDim.x) {
        int bi, bj;
        tile_of(tiles, turn, bi, bj);
        const int i0 = bi * BM, j0 = bj * BN;
        v16i acc[TI][2];
#pragma unroll
        for (int ti = 0; ti < TI; ++ti)
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[ti][w][e] = 0;
        v4i fp[2][TI], fw[2][2];
        auto fragments = [&](int set, const int8_t* from, int ks) {
#pragma unroll
            for (int ti = 0; ti < TI; ++ti) fp[set][ti] = *(const v4i*)(from + swizzled(wm * (BM / WM) + ti * 32 + lr, ks * 2 + lh));
#pragma unroll
            for (int w = 0; w < 2; ++w) fw[set][w] = *(const v4i*)(from + BM * 128 + swizzled(w * BN + wn * 32 + lr, ks * 2 + lh));
        };
        auto multiply = [&](int set) {
#pragma unroll
            for (int ti = 0; ti < TI; ++ti)
#pragma unroll
                for (int w = 0; w < 2; ++w) acc[ti][w] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[set][w], fp[set][ti], acc[ti][w], 0, 0, 0);
        };
        if (!prefetched) {
            operands(bi, bj);
            issue(0, 0);
        }
        if (nk > 1) issue(1, 1);
        if (!prefetched) {   // (a step that was fetched ahead is there: see below)
            if (nk > 1) wait_copies<CH>();
            else wait_copies<0>();
            __builtin_amdgcn_s_barrier();
        }
        fragments(0, lds, 0);
        int cur = 0;
        for (int kt = 0; kt < nk; ++kt) {
            const int8_t* const from = lds + cur * STAGE;
            const int8_t* const next = lds + (cur ^ 1) * STAGE;
#pragma unroll
            for (int u = 0; u < 3; ++u) {
                fragments((u + 1) & 1, from, u + 1);
                multiply(u & 1);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            wait_copies<0>();
            __builtin_amdgcn_s_barrier();
            // this step's stage is free, the next step's is full
            if (early && kt + 2 < nk) issue(kt + 2, cur);
            if (kt + 1 < nk) fragments(0, next, 0);
            multiply(1);
            if (!early && kt + 2 < nk) issue(kt + 2, cur);
            cur ^= 1;
        }
        // Nobody reads a stage any more: the first one takes the next tile's first step, the second one the staging.
        const int after = turn + (int)gridDim.x;
        prefetched = after < tiles.all;
        if (prefetched) {
            int ni, nj;
            tile_of(tiles, after, ni, nj);
            operands(ni, nj);
            issue(0, 0);
        }
        const bool edge = j0 + BN > a.n;
        const int jw = j0 + wn * 32, block = jw >> 5;   // this wavefront's columns
        int8_t* const mine = lds + STAGE + wave * STAGED;
        bool waited = false;
#pragma unroll
        for (int ti = 0; ti < TI; ++ti) {
            const int iw = i0 + wm * (BM / WM) + ti * 32, i = iw + lr;
            float g[16], u[16], good = 0;
            uint32_t top_g = 0, top_u = 0;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                g[e] = (float)acc[ti][0][e] * sc;
                u[e] = (float)acc[ti][1][e] * sc;
            }
            if (edge)   // columns beyond the matrix are no part of a block (their sums are zero, but the scale may be anything)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (jw + 8 * (e >> 2) + 4 * lh + (e & 3) >= a.n) g[e] = u[e] = 0.0f;
            if (a.g.q) {
                // the largest magnitude is that of the largest sum: rounding and the scale keep their order (an infinite scale leaves no block finite, either way)
                top_g = abs_max16(acc[ti][0], sc);
                top_u = abs_max16(acc[ti][1], sc);
                const uint32_t eg = ckpt_exponent(top_g), eu = ckpt_exponent(top_u);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    *(uint32_t*)(mine + 32 * YROW + lr * QROW + 8 * q + 4 * lh) = codes4(g + 4 * q, top_g, eg);
                    *(uint32_t*)(mine + 32 * (YROW + QROW) + lr * QROW + 8 * q + 4 * lh) = codes4(u + 4 * q, top_u, eu);
                }
                top_g = eg;
                top_u = eu;
            }
            gate<T>(a.act, g, u, u);
#pragma unroll
            for (int e = 0; e < 16; ++e) good = __builtin_fmaf(u[e], u[e], good);   // (zero beyond the matrix)
#pragma unroll
            for (int q = 0; q < 4; ++q) stage4((T*)(mine + lr * YROW) + 8 * q + 4 * lh, u + 4 * q);
            good += __shfl_xor(good, 32);
            wave_lds_fence();
            if (prefetched && !waited) {   // copies and stores complete in issue order: before the first store
                wait_copies<0>();
                waited = true;
            }
            if (jw < a.n) {
                if (a.good && lh == 0 && i < a.rows) a.good[(int64_t)block * a.rows + i] = good;
                constexpr int PER = 16 / (int)sizeof(T), LANES = 32 / PER, ROWS = 64 / LANES;   // elements of a store, lanes and rows of an instruction
#pragma unroll
                for (int r0 = 0; r0 < 32; r0 += ROWS) {
                    const int r = r0 + lane / LANES, c = lane % LANES * PER, n = a.n - (jw + c);
                    const T* const from = (const T*)(mine + r * YROW) + c;
                    if (iw + r < a.rows && n > 0) {
                        T* const to = (T*)a.y + ((int64_t)(iw + r) * a.ldy + jw + c);
                        const u32x4 v = *(const u32x4*)from;
                        if (n >= PER) write_as<u32x4>(to, v);
                        else
                            for (int e = 0; e < PER - 1; ++e)
                                if (e < n) to[e] = from[e];
                    }
                }
            }
            if (a.g.q) {
                const int r = lane >> 1, at = jw + 16 * (lane & 1);   // two lanes to a row's 32 codes
                if (iw + r < a.rows && at < (int)a.g.pitch) {
                    *(u32x4*)(a.g.q + (int64_t)(iw + r) * a.g.pitch + at) = *(const u32x4*)(mine + 32 * YROW + r * QROW + 16 * (lane & 1));
                    *(u32x4*)(a.u.q + (int64_t)(iw + r) * a.u.pitch + at) = *(const u32x4*)(mine + 32 * (YROW + QROW) + r * QROW + 16 * (lane & 1));
                }
                if (i < a.rows) {
                    uint8_t* const eg = a.g.e + (int64_t)i * a.g.epitch;
                    uint8_t* const eu = a.u.e + (int64_t)i * a.u.epitch;
                    if (lh == 0 && block < a.g.blocks) {
                        eg[block] = (uint8_t)top_g;
                        eu[block] = (uint8_t)top_u;
                    }
                    if (bj == tiles.j - 1 && wn == 0) {   // the pads behind the last tile
                        for (int at = j0 + BN + 16 * lh; at < (int)a.g.pitch; at += 32) {
                            *(u32x4*)(a.g.q + (int64_t)i * a.g.pitch + at) = u32x4{0, 0, 0, 0};
                            *(u32x4*)(a.u.q + (int64_t)i * a.u.pitch + at) = u32x4{0, 0, 0, 0};
                        }
                        for (int at = a.g.blocks + lh; at < (int)a.g.epitch; at += 2) eg[at] = eu[at] = 0;
                    }
                }
            }
            wave_lds_fence();   // (the next rows' values go where these lie)
        }
        // Every wavefront has waited for its copies of the next tile's first step: they are there for all behind this barrier.  And for what it staged, also where it has no
        // columns or rows to read back: the next tile's second step goes where that lies.
        if (prefetched) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
        }
    }
}

// ------------------------------------------------------------------------------------------------
// Up to 16 rows, nothing kept (serving): tiles of 16 outputs, eight wavefronts that share out the reduction.  What counts is that the weights stream in:
// lanes load what they multiply themselves, 16 bytes of a row each, and all of a wavefront's loads of up to 512 bytes of every row are under way at once.
// 1 x 4096 x 4096: 34 MB of weights in 6.6 us (5.1 TB/s), and 2.6 for the sums of the goodness; by tiles of 32 x 32 12 in all, where only half as many workgroups read.
// ------------------------------------------------------------------------------------------------
constexpr int ROW_WAVES = 8, ROW_STEPS = 8;   // wavefronts, steps of 64 bytes under way

template <typename T> __global__ __launch_bounds__(ROW_WAVES * 64) void k_gated_rows(GatedArgs a, int ntiles, int per_xcd)
{
    __shared__ __attribute__((aligned(16))) v4i part[ROW_WAVES][2][64];
    const int t = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
    if (t >= ntiles) return;
    const int j0 = t * 16, jrows = min(16, a.n - j0);
    const int lane = threadIdx.x & 63, l16 = lane & 15, lk = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kpad = (a.k + 15) & ~15, nk = (kpad + 63) >> 6, per = (nk + ROW_WAVES - 1) / ROW_WAVES;
    const int k0 = wave * per, k1 = min(nk, k0 + per);   // this wavefront's steps
    const __amdgpu_buffer_rsrc_t rp = __builtin_amdgcn_make_buffer_rsrc((void*)a.a_q, 0, (int)(a.rows * a.ld), 0x00020000);
    const __amdgpu_buffer_rsrc_t rg = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w_q + (int64_t)j0 * a.ld), 0, (int)(jrows * a.ld), 0x00020000);
    const __amdgpu_buffer_rsrc_t ru = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w_q + (int64_t)(a.n + j0) * a.ld), 0, (int)(jrows * a.ld), 0x00020000);
    const int row = l16 * (int)a.ld + lk * 16;
    v4i ag = {0, 0, 0, 0}, au = {0, 0, 0, 0};
    for (int k = k0; k < k1; k += ROW_STEPS) {
        v4i p[ROW_STEPS], g[ROW_STEPS], u[ROW_STEPS];
#pragma unroll
        for (int s = 0; s < ROW_STEPS; ++s) {
            const int at = (k + s) * 64 + lk * 16, off = k + s < k1 && at < kpad ? row + (k + s) * 64 : 0x7FFFFFF0;
            g[s] = (v4i)__builtin_amdgcn_raw_buffer_load_b128(rg, off, 0, 0);
            u[s] = (v4i)__builtin_amdgcn_raw_buffer_load_b128(ru, off, 0, 0);
            p[s] = (v4i)__builtin_amdgcn_raw_buffer_load_b128(rp, off, 0, 0);
        }
#pragma unroll
        for (int s = 0; s < ROW_STEPS; ++s) {
            ag = __builtin_amdgcn_mfma_i32_16x16x64_i8(g[s], p[s], ag, 0, 0, 0);
            au = __builtin_amdgcn_mfma_i32_16x16x64_i8(u[s], p[s], au, 0, 0, 0);
        }
    }
    part[wave][0][lane] = ag;
    part[wave][1][lane] = au;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    // lane: sample l16, outputs 4 lk .. + 3
#pragma unroll
    for (int w = 1; w < ROW_WAVES; ++w) {
        ag += part[w][0][lane];
        au += part[w][1][lane];
    }
    const int j = j0 + 4 * lk;
    const float sc = a.s_a[0] * a.s_w[0];
    float g[4], u[4], y[4], s = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        g[e] = (float)ag[e] * sc;
        u[e] = (float)au[e] * sc;
    }
    gate<T>(a.act, g, u, y);
    if (l16 < a.rows && j < a.n) store4((T*)a.y + ((int64_t)l16 * a.ldy + j), a.n - j, y);
    if (a.good) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s = j + e < a.n ? __builtin_fmaf(y[e], y[e], s) : s;
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        if (lane < a.rows) a.good[(int64_t)t * a.rows + lane] = s;   // (lane < 16)
    }
}

// goodness[row] = sum of its parts: 32 rows of a workgroup, every eighth part a thread
__global__ __launch_bounds__(256) void k_gated_goodness(const float* part, float* goodness, int32_t rows, int32_t parts)
{
    __shared__ float red[8][32];
    const int r = threadIdx.x & 31, lane = threadIdx.x >> 5, row = (int)blockIdx.x * 32 + r;
    float s = 0;
    if (row < rows)
#pragma unroll 8
        for (int p = lane; p < parts; p += 8) s += part[(int64_t)p * rows + row];
    red[lane][r] = s;
    __syncthreads();
    if (lane == 0 && row < rows) {
        for (int p = 1; p < 8; ++p) s += red[p][r];
        goodness[row] = s;
    }
}

// ------------------------------------------------------------------------------------------------
// launches
// ------------------------------------------------------------------------------------------------
static int64_t gated_parts(int64_t rows, int64_t n) { return rows <= 16 ? (n + 15) / 16 : (n + 31) / 32; }   // of a row's goodness, at most
size_t gated_workspace(int64_t rows, int64_t n, int64_t)
{
    return align_up(std::max<size_t>((size_t)(rows * gated_parts(rows, n)) * sizeof(float), FF_WS_MIN_BYTES), 16);
}

template <typename T, int BM, int BN, int WM, int WN> static void tiles_launch(const GatedArgs& a, int per_unit, hipStream_t s)
{
    GatedTiles t = {};
    t.i = (a.rows + BM - 1) / BM;
    t.j = (a.n + BN - 1) / BN;
    t.all = t.i * t.j;
    t.per_turn = (std::min(t.all, num_cus() * per_unit) + 7) / 8;
    k_gated_tiles<T, BM, BN, WM, WN><<<(unsigned)(8 * t.per_turn), WM * WN * 64, 0, s>>>(a, t);
}

// Which kernel, by what was measured (us; bf16, kept, samples x inputs x outputs; 32 x 32 tiles, 128 x 64, 256 x 128):
//   up to four 32 x 32 tiles for a compute unit: 512 x 784 x 2000 11.2 10.6 19.8, 256 x 4096 x 4096 24.5 27.6 46.5; twice as many: 1024 x 784 x 2000 18.2 12.0 20.0
//   beyond, whichever takes fewer rounds of the chip's tiles, one of 256 x 128 counting as 1.75 of 128 x 64, two of which share a compute unit:
//   2048 x 784 x 2000 33 16.6 22.0, 2048 x 4096 x 4096 181 89 72, 4096 x 2000 x 2000 100 46 40, 6000 x 2000 x 2000 142 65 71, 8192 x 2000 x 2000 191 84 73, 16384 x 64 x 1024 65 28 26
enum GatedKernel { GATED_ROWS, GATED_FEW, GATED_MIDDLE, GATED_LARGE };
static GatedKernel gated_kernel(int64_t rows, int64_t n, bool kept)
{
    if (rows <= 16 && !kept) return GATED_ROWS;
    const int64_t cus = num_cus(), few = ((rows + 31) / 32) * ((n + 31) / 32);
    if (few <= 4 * cus) return GATED_FEW;
    const int64_t middle = ((rows + 127) / 128) * ((n + 63) / 64), large = ((rows + 255) / 256) * ((n + 127) / 128);
    return 7 * ((large + cus - 1) / cus) < 4 * ((middle + 2 * cus - 1) / (2 * cus)) ? GATED_LARGE : GATED_MIDDLE;
}

template <typename T> static hipError_t forward_of(GatedArgs a, float* goodness, hipStream_t s)
{
    const GatedKernel which = gated_kernel(a.rows, a.n, a.g.q != nullptr);
    const int64_t parts = which == GATED_ROWS ? (a.n + 15) / 16 : (a.n + 31) / 32, ntiles = (int64_t)((a.rows + 31) / 32) * parts;
    const int per_xcd = (int)((ntiles + 7) / 8);
    if (goodness && parts == 1) a.good = goodness;
    switch (which) {
        case GATED_ROWS: k_gated_rows<T><<<(unsigned)(8 * per_xcd), ROW_WAVES * 64, 0, s>>>(a, (int)ntiles, per_xcd); break;
        case GATED_FEW: k_gated_few<T><<<(unsigned)(8 * per_xcd), WAVES * 64, 0, s>>>(a, (int)ntiles, per_xcd); break;
        case GATED_MIDDLE: tiles_launch<T, 128, 64, 2, 2>(a, 2, s); break;
        case GATED_LARGE: tiles_launch<T, 256, 128, 2, 4>(a, 1, s); break;
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (goodness && parts > 1) k_gated_goodness<<<(unsigned)((a.rows + 31) / 32), 256, 0, s>>>(a.good, goodness, a.rows, (int32_t)parts);
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
