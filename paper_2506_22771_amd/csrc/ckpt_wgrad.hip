// Weight gradient of a linear layer from the 8-bit checkpoint of its input:
//
//     dW[n][k] = gamma[k] S[n][k] + beta[k] db[n],   S[n][k] = sum over rows m of dy[m][n] x[m][k],   db[n] = sum over rows m of dy[m][n]
//
// x is what the checkpoint stands for.  Behind a layer norm that is the normalised row h, and gamma, beta are the norm's parameters: the layer's
// input gamma h + beta is never kept, its share of the gradient follows from the two sums.
//
// The products run on bf16 matrix instructions with fp32 accumulators.  A checkpoint's value q 2^s is exact in bf16.  dy is taken as one (bf16), two
// (fp16) or three (fp32) bf16 terms, split by truncation, so that their sum is dy exactly (what lies below 2^-126 aside) and every product is exact: the only
// roundings are those of the fp32 sums, as in a product of fp32 matrices, of which this is several times the rate.
//
// A workgroup owns BT x BT outputs and walks over the rows in steps of BM.  Both operands lie in memory with the reduction (m)
// as the slow axis.  A step's BM x BT elements go through registers, which is where codes become bf16 and dy its terms, into LDS as
// they lie, and the fragments are read with the transposing LDS read.  Three stages of LDS: while a step is multiplied the one after the next is
// written and the first fragments of the next are read already, so that no wavefront waits for LDS behind the barrier; registers hold the step after those.
//
// Bound by the matrix pipe and, in the large case, by what the card sustains of it.  Measured: 16384 rows, 4096 x 4096, bf16 511 to 560 us, 0.98 to
// 1.08 PFLOP/s (a library product of bf16 matrices, both in memory already, 513 to 560); 2048 rows, 2000 x 2000, fp32 72 to 77 us, of which 12 add the splits: 0.68
// PFLOP/s of the three bf16 products (a library product of fp32 matrices 123, one of bf16 matrices 29); 128 rows, 500 x 784, fp32 7.5: 104
// workgroups of 64 x 64 outputs on 256 compute units, four steps one after the other.
#include <type_traits>

#include "ckpt.hpp"
#include "norm.hpp"
#include "wgrad_plan.hpp"

namespace ffi {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

template <typename T> struct Terms;
template <> struct Terms<bf16_t> { static constexpr int N = 1; };
template <> struct Terms<f16_t> { static constexpr int N = 2; };
template <> struct Terms<float> { static constexpr int N = 3; };
// Rows of a step: three stages of all terms and the checkpoint's values in LDS, which two workgroups share where tiles are small.
template <typename T, int BT> constexpr int step_rows() { return Terms<T>::N == 3 && BT > 64 ? 16 : 32; }

struct WgradArgs {
    const void* dy;
    int64_t lddy;
    CkptPtr c;
    int64_t rows;
    int32_t n, k, tiles_n, tiles_k, splits;
    int64_t steps, per;      // steps of all rows, steps of a split
    int64_t plain;           // steps before this one are read with the range check alone
    const void* gamma;
    const void* beta;
    int32_t param_kind;      // type of gamma and beta
    float* dw;
    float* db;
    int32_t accumulate;
    float* part;             // splits > 1: a split's dw and db, `stride` apart
    int64_t stride;
};

__device__ __forceinline__ float param_at(const void* p, int kind, int64_t at, float none)
{
    if (!p) return none;
    if (kind == FF_F32) return ((const float*)p)[at];
    const uint32_t w = ((const uint16_t*)p)[at];
    return kind == FF_BF16 ? bf16_value(w) : (float)__builtin_bit_cast(_Float16, (uint16_t)w);
}

// Transposing LDS read of 16-bit elements: each group of 16 lanes reads four rows of 32 bytes (lanes 4r .. 4r + 3 give the
// quarters of row r) and lane j of the group receives column j, rows 0 .. 3.
__device__ __forceinline__ v4s tr_read16(const char* p)
{
    typedef __attribute__((address_space(3))) v4s* lds_ptr;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p);
}
// Chunk (16 bytes, eight elements) c of row m lies at c ^ swizzle(m): the eight rows of 64 bytes that one transposing read of a wavefront takes
// then fall into different banks.
template <int BT> __device__ __forceinline__ int swizzle(int m)
{
    return BT == 256 ? ((m & 3) | ((m >> 1) & 4)) << 2 : BT == 128 ? (m & 3) << 2 : ((m >> 1) & 1) << 2;
}

// The bf16 terms of eight values of dy: t0 + t1 + t2, each the leading bits of what the ones before leave (truncated, which is exact: 24 bits are three
// times eight).  Infinities stay in the first term alone; a NaN is one in one of the terms.
__device__ __forceinline__ void terms_of(const Raw8<bf16_t>& r, u32x4 t[1]) { t[0] = r.a; }
__device__ __forceinline__ uint32_t high_pair(float lo, float hi) { return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u); }
__device__ __forceinline__ float lead_of(float v) { return __uint_as_float(__float_as_uint(v) & 0xFFFF0000u); }
__device__ __forceinline__ float rest_of(float v) { return __builtin_fabsf(v) == __builtin_inff() ? 0.0f : v - lead_of(v); }
__device__ __forceinline__ void terms_of(const Raw8<f16_t>& r, u32x4 t[2])
{
    float v[8];
    raw_values(r, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        t[0][i] = high_pair(v[2 * i], v[2 * i + 1]);
        t[1][i] = high_pair(rest_of(v[2 * i]), rest_of(v[2 * i + 1]));
    }
}
__device__ __forceinline__ void terms_of(const Raw8<float>& r, u32x4 t[3])
{
    float v[8];
    raw_values(r, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = v[2 * i], b = v[2 * i + 1], a1 = rest_of(a), b1 = rest_of(b);
        t[0][i] = high_pair(a, b);
        t[1][i] = high_pair(a1, b1);
        t[2][i] = high_pair(a1 - lead_of(a1), b1 - lead_of(b1));   // (finite or NaN)
    }
}

// v + the sum of eight bf16 values
__device__ __forceinline__ float sum_of(v8bf f, float v)
{
    const v2bf one = {(__bf16)1.0f, (__bf16)1.0f};
    v = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(f, f, 0, 1), one, v, false);
    v = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(f, f, 2, 3), one, v, false);
    v = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(f, f, 4, 5), one, v, false);
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(f, f, 6, 7), one, v, false);
}

// f(0), ..., f(N - 1), as constants
template <int I, int N, typename F> __device__ __forceinline__ void each_of(F&& f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>());
        each_of<I + 1, N>(f);
    }
}

// Two by WK wavefronts.
template <typename T, int BT, int WK> struct WgradTile {
    static constexpr int P = Terms<T>::N, BM = step_rows<T, BT>();
    static constexpr int THREADS = 128 * WK;
    static constexpr int CPR = BT / 8;                   // chunks of a row
    static constexpr int CH = BM * CPR / THREADS;        // chunks of a thread, of each operand
    static constexpr int ROWS = THREADS / CPR;           // rows between a thread's chunks
    static constexpr int PLANE = BM * BT * 2;            // bytes of one term
    static constexpr int STAGE = (P + 1) * PLANE;
    static constexpr int SUB = BM / 16;                  // matrix instructions along a step
    static_assert(WK >= BT / 64 || BT / 64 == 1, "sums of dy");
    static constexpr int TI = BT / 64, TJ = BT / (32 * WK);   // a wavefront's outputs, in tiles of 32
    static constexpr int PIECES = SUB * P * TI;          // a wavefront's fragments of dy in a step, TJ matrix instructions each
    static constexpr int EVERY = PIECES / CH;            // pieces to a chunk
    // Steps on their way in registers: as many as a step's matrix instructions (32 clocks each) need to cover some 2500 clocks.
    static constexpr int SETS = BT == 256 ? 2 : 4;
    // Fragments of dy read ahead: a read takes some 130 clocks and more, a piece 32 TJ of its SIMD's matrix pipe.
    static constexpr int AHEAD = PIECES < 3 ? 2 : BT == 256 ? 2 : 3;
    static constexpr int LDS = 3 * STAGE;
    static_assert(CH >= 1 && LDS <= 160 * 1024 && ROWS % 8 == 0 && PIECES % CH == 0 && TJ <= TI, "tile");
};

template <typename T, int BT, int WK>
__global__ __launch_bounds__(128 * WK) __attribute__((amdgpu_waves_per_eu(BT == 256 ? WK / 2 : 2))) void k_ckpt_wgrad(WgradArgs a)
{
    using S = WgradTile<T, BT, WK>;
    __shared__ __attribute__((aligned(16))) char lds[S::LDS];
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wn = wave / WK, wk = wave % WK;
    // Workgroups go to the eight XCDs in turn: each takes consecutive tiles, in bands of four tiles of n, so that its L2 holds few panels.
    const int items = a.tiles_n * a.tiles_k * a.splits, per_xcd = (items + 7) >> 3;
    const int item = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
    if (item >= items) return;   // (uniform)
    const int tiles = a.tiles_n * a.tiles_k, split = item / tiles, tile = item - split * tiles;
    const int band = tile / (4 * a.tiles_k), in_band = tile - band * 4 * a.tiles_k, height = min(4, a.tiles_n - 4 * band);
    const int tk = in_band / height, tn = 4 * band + in_band - tk * height;
    const int n0 = tn * BT, k0 = tk * BT;
    const int64_t step0 = split * a.per, step1 = min(step0 + a.per, a.steps);

    // This thread's chunk column, and rows r0, r0 + ROWS, ...  Columns that do not exist are read as some that do: their outputs are not stored.
    const int cc = tid % S::CPR, r0 = tid / S::CPR;
    const int cn = min(n0 + 8 * cc, (a.n - 1) & ~7);
    const int64_t ck = min((int64_t)(k0 + 8 * cc), a.c.pitch - 8);
    const int cb = min((k0 + 8 * cc) >> 5, a.c.blocks - 1);
    const T* const dy = (const T*)a.dy + cn;
    const int8_t* const cq = a.c.q + ck;
    const uint8_t* const ce = a.c.e + cb;
    struct Chunk { Raw8<T> d; u32x2 q; uint32_t e; };
    // Steps in order, from scalar bases and this thread's fixed offsets.  A chunk of dy may reach into the next row (n not a multiple of
    // eight); words beyond the end of a matrix, rows that do not exist among them, fail the buffer's range check and are zero.  All of an address that
    // can pass the end is in the vector offset: the scalar offset is no part of what is compared with the size, and may be larger than it in a step of few rows.
    const uint32_t off_d = (uint32_t)(r0 * a.lddy + cn) * sizeof(T), off_q = (uint32_t)(r0 * a.c.pitch + ck), off_e = (uint32_t)(r0 * a.c.epitch) + cb;
    const int64_t step_d = S::BM * a.lddy * (int64_t)sizeof(T), step_q = S::BM * a.c.pitch, step_e = S::BM * a.c.epitch;
    const char *base_d = (const char*)a.dy + step0 * step_d, *base_q = (const char*)a.c.q + step0 * step_q, *base_e = (const char*)a.c.e + step0 * step_e;
    int64_t left_d = ((a.rows - 1) * a.lddy + a.n) * (int64_t)sizeof(T) - step0 * step_d;   // bytes up to the end
    int64_t left_q = a.rows * a.c.pitch - step0 * step_q, left_e = a.rows * a.c.epitch - step0 * step_e;
    auto buffer = [](const char* base, int64_t left) {
        return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)min(left, (int64_t)0x7FFFFFFF), 0x00020000);
    };
    auto fetch = [&](int i) {
        const __amdgpu_buffer_rsrc_t bd = buffer(base_d, left_d), bq = buffer(base_q, left_q), be = buffer(base_e, left_e);
        const uint32_t at_d = off_d + (uint32_t)(i * S::ROWS * a.lddy * (int64_t)sizeof(T)), at_q = off_q + (uint32_t)(i * S::ROWS * a.c.pitch),
                       at_e = off_e + (uint32_t)(i * S::ROWS * a.c.epitch);
        Chunk c;
        c.d.a = __builtin_amdgcn_raw_buffer_load_b128(bd, (int)at_d, 0, 0);
        if constexpr (sizeof(T) == 4) c.d.b = __builtin_amdgcn_raw_buffer_load_b128(bd, (int)(at_d + 16), 0, 0);
        c.q = __builtin_amdgcn_raw_buffer_load_b64(bq, (int)at_q, 0, 0);
        c.e = __builtin_amdgcn_raw_buffer_load_b8(be, (int)at_e, 0, 0);
        return c;
    };
    auto advance = [&](bool more) {   // to the next step, or not beyond the last (which is then fetched again and used by nobody)
        const int64_t d = more ? step_d : 0, q = more ? step_q : 0, e = more ? step_e : 0;
        base_d += d;
        left_d -= d;
        base_q += q;
        left_q -= q;
        base_e += e;
        left_e -= e;
    };
    // Rows that do not exist are zero in both operands, columns beyond n too.
    auto fetch_last = [&](int64_t step, int i) {
        const int64_t m = step * S::BM + r0 + i * S::ROWS;
        Chunk c = {{}, {0, 0}, 0};
        if (m < a.rows) c = Chunk{load_raw(dy + m * a.lddy, min(8, a.n - cn)), *(const u32x2*)(cq + m * a.c.pitch), ce[m * a.c.epitch]};
        return c;
    };
    auto put = [&](char* stage, int i, Chunk c) {
        opaque(c.d);
        opaque(c.q);
        opaque(c.e);
        const int m = r0 + i * S::ROWS;
        char* const at = stage + m * (BT * 2) + ((cc ^ swizzle<BT>(m)) << 4);
        u32x4 t[S::P];
        terms_of(c.d, t);
#pragma unroll
        for (int p = 0; p < S::P; ++p) *(u32x4*)(at + p * S::PLANE) = t[p];
        float v[8];
        ckpt_values(c.q, c.e, v);
        u32x4 x;
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = high_pair(v[2 * u], v[2 * u + 1]);   // (exact)
        *(u32x4*)(at + S::P * S::PLANE) = x;
    };

    float gamma[S::TJ], beta[S::TJ];   // of this lane's columns, asked for before the loop
#pragma unroll
    for (int j = 0; j < S::TJ; ++j) {
        const int k = min(k0 + 32 * (wk * S::TJ + j) + lr, a.k - 1);
        gamma[j] = param_at(a.gamma, a.param_kind, k, 1.0f);
        beta[j] = param_at(a.beta, a.param_kind, k, 0.0f);
    }
    v16f acc[S::TI][S::TJ];
    float db = 0;   // this lane's share of the sums of dy, for the tile wk % TI of its wavefront's rows n
#pragma unroll
    for (int i = 0; i < S::TI; ++i)
#pragma unroll
        for (int j = 0; j < S::TJ; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
    // A lane's place in a transposing read: row 8 lh + (lane & 15) / 4 of a 16-row piece (and four rows on for the second half of a fragment, where
    // the swizzle is the same), columns 16 ((lane >> 4) & 1) + 4 (lane & 3) of a 32-column tile.
    const int tr_row = 8 * lh + ((lane & 15) >> 2), tr_at = tr_row * (BT * 2) + ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) << 4) + 8 * (lane & 1);
    int at_n[S::TI], at_k[S::TJ];
#pragma unroll
    for (int i = 0; i < S::TI; ++i) at_n[i] = tr_at + ((((wn * S::TI + i) << 2) ^ swizzle<BT>(tr_row)) << 4);
    const int at_sum = tr_at + ((((wn * S::TI + wk % S::TI) << 2) ^ swizzle<BT>(tr_row)) << 4);
#pragma unroll
    for (int j = 0; j < S::TJ; ++j) at_k[j] = tr_at + ((((wk * S::TJ + j) << 2) ^ swizzle<BT>(tr_row)) << 4) + S::P * S::PLANE;
    auto fragment = [&](const char* stage, int at, int more) {   // more: a constant
        const v4s lo = tr_read16(stage + at + more), hi = tr_read16(stage + at + more + 4 * BT * 2);
        return __builtin_bit_cast(v8bf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto fragment_n = [&](const char* stage, int piece) {
        const int i = piece % S::TI, p = piece / S::TI % S::P, s = piece / (S::TI * S::P);
        return fragment(stage, at_n[i], s * 16 * BT * 2 + p * S::PLANE);
    };
    auto meet = [&] {   // this wavefront's LDS operations are done, then everybody's; loads from memory stay on their way
        wait_lds();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    const int64_t plain = min(step1, a.plain);
    if (step0 < plain) {
        constexpr int SETS = S::SETS;
        Chunk c[SETS][S::CH];
        int64_t fetched = step0;  // the step that fetch() reads
        auto fetch_step = [&](Chunk* to) {
#pragma unroll
            for (int i = 0; i < S::CH; ++i) to[i] = fetch(i);
            advance(fetched + 1 < plain);
            ++fetched;
        };
        // The first steps are all asked for before any is waited for; two go to LDS and make room for two more.
#pragma unroll
        for (int st = 0; st < SETS; ++st) fetch_step(c[st]);
#pragma unroll
        for (int st = 0; st < 2; ++st) {
#pragma unroll
            for (int i = 0; i < S::CH; ++i) put(lds + st * S::STAGE, i, c[st][i]);
            fetch_step(c[st]);
        }
        meet();
        char *now = lds, *next = lds + S::STAGE, *after = lds + 2 * S::STAGE;
        v8bf fa[S::AHEAD], fb[S::TJ];
#pragma unroll
        for (int i = 0; i < S::AHEAD; ++i) fa[i] = fragment_n(now, i);
#pragma unroll
        for (int j = 0; j < S::TJ; ++j) fb[j] = fragment(now, at_k[j], 0);
        v8bf fb_next[S::TJ];
        v8bf fs;
        auto work = [&](auto set) {
            constexpr int ST = (decltype(set)::value + 2) % SETS;   // (the first two sets hold later steps than the others)
#pragma unroll
            for (int piece = 0; piece < S::PIECES; ++piece) {
                const int i = piece % S::TI, p = piece / S::TI % S::P, s = piece / (S::TI * S::P), chunk = piece / S::EVERY;
                if (piece % (S::TI * S::P) == 0) {   // the next sixteen rows' fragments of k
#pragma unroll
                    for (int j = 0; j < S::TJ; ++j)
                        fb_next[j] = s + 1 < S::SUB ? fragment(now, at_k[j], (s + 1) * 16 * BT * 2) : fragment(next, at_k[j], 0);
                }
                const v8bf f = fa[0];
#pragma unroll
                for (int d = 0; d + 1 < S::AHEAD; ++d) fa[d] = fa[d + 1];
                constexpr int AT = S::PIECES - S::AHEAD;
                fa[S::AHEAD - 1] = piece < AT ? fragment_n(now, piece + S::AHEAD) : fragment_n(next, piece - AT);
                if (S::TI > 1 && i == 0) fs = fragment(now, at_sum, s * 16 * BT * 2 + p * S::PLANE);
#pragma unroll
                for (int j = 0; j < S::TJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, fb[j], acc[i][j], 0, 0, 0);
                if (i == S::TI - 1) {
                    db += sum_of(S::TI > 1 ? fs : f, 0.0f);
                    opaque(db);
                }
                if (piece % S::EVERY == 0) {
                    put(after, chunk, c[ST][chunk]);
                    c[ST][chunk] = fetch(chunk);
                }
                if ((piece + 1) % (S::TI * S::P) == 0) {
#pragma unroll
                    for (int j = 0; j < S::TJ; ++j) fb[j] = fb_next[j];
                }
                if (piece % S::EVERY == S::EVERY - 1) {
                    // What is to run beside a matrix instruction has to stand behind it, before the next one.
#pragma unroll
                    for (int m = 0; m < S::EVERY * S::TJ; ++m) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // matrix
                        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);   // LDS reads
                        __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);   // vector arithmetic
                        __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);   // LDS writes
                        __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);   // loads
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            advance(fetched + 1 < plain);
            ++fetched;
            meet();
            char* const first = now;
            now = next;
            next = after;
            after = first;
        };
        // (Whole rounds without a branch in them: where a step may be left out the compiler counts on the fewest loads under way and
        // waits for nearly all of them.)
        int64_t step = step0;
        for (; step + SETS <= plain; step += SETS) each_of<0, SETS>(work);
        each_of<0, SETS - 1>([&](auto st) {
            if (step + decltype(st)::value < plain) work(st);
        });
    }
    // what is left: the step with the last row where that ends inside a word (the range check goes by words), or all of them where rows lie too far apart
    for (int64_t step = max(step0, plain); step < step1; ++step) {
        meet();
#pragma nounroll
        for (int i = 0; i < S::CH; ++i) put(lds, i, fetch_last(step, i));
        meet();
#pragma nounroll
        for (int s = 0; s < S::SUB; ++s) {
            v8bf fb[S::TJ];
#pragma unroll
            for (int j = 0; j < S::TJ; ++j) fb[j] = fragment(lds + s * 16 * BT * 2, at_k[j], 0);
#pragma unroll
            for (int piece = 0; piece < S::P * S::TI; ++piece) {
                const int i = piece % S::TI;
                const v8bf fa = fragment_n(lds + s * 16 * BT * 2, piece);
#pragma unroll
                for (int j = 0; j < S::TJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa, fb[j], acc[i][j], 0, 0, 0);
                if (i == wk % S::TI) db += sum_of(fa, 0.0f);
            }
        }
    }
    meet();

    // sums of dy, in LDS (which nothing reads any more): both halves of a wavefront have eight of sixteen rows
    float* const sums = (float*)lds;
    db += __shfl_xor(db, 32);
    if (lh == 0 && wk < S::TI) sums[32 * (wn * S::TI + wk) + lr] = db;
    __syncthreads();
    const bool whole = a.splits == 1, add = whole && a.accumulate;
    float* const out = whole ? a.dw : a.part + (int64_t)split * a.stride;
    float* const out_db = whole ? a.db : a.part + (int64_t)split * a.stride + (int64_t)a.n * a.k;
    if (tk == 0 && out_db && tid < BT && n0 + tid < a.n) out_db[n0 + tid] = add ? out_db[n0 + tid] + sums[tid] : sums[tid];
    // Both parts of the result are linear in the rows: gamma and beta are applied to every split's sums.
#pragma unroll
    for (int j = 0; j < S::TJ; ++j) {
        const int k = k0 + 32 * (wk * S::TJ + j) + lr;
        if (k >= a.k) continue;
#pragma unroll
        for (int i = 0; i < S::TI; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int nl = 32 * (wn * S::TI + i) + (v & 3) + 8 * (v >> 2) + 4 * lh, n = n0 + nl;
                if (n >= a.n) continue;
                float r = gamma[j] * acc[i][j][v];
                if (a.beta) r = __builtin_fmaf(beta[j], sums[nl], r);
                float* const to = out + (int64_t)n * a.k + k;
                *to = add ? *to + r : r;
            }
    }
}

// Adds the splits' results in order, four values a thread and round: dw, then db.  No splits (no rows): zero.
__global__ __launch_bounds__(256) void k_ckpt_wgrad_sum(WgradArgs a)
{
    const int64_t size = (int64_t)a.n * a.k, end = size + (a.db ? a.n : 0);
    for (int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; at < end; at += (int64_t)gridDim.x * 1024) {
        float4 v = make_float4(0, 0, 0, 0);
        const float* p = a.part + at;   // (a split's results are followed by room up to `stride`, a multiple of four)
#pragma unroll 4
        for (int s = 0; s < a.splits; ++s, p += a.stride) {
            const float4 t = *(const float4*)p;
            v = make_float4(v.x + t.x, v.y + t.y, v.z + t.z, v.w + t.w);
        }
        const float r[4] = {v.x, v.y, v.z, v.w};
        if (at + 4 <= size) {
            float* const to = a.dw + at;
            u32x4 o;
            if (a.accumulate) o = read_as<u32x4>(to);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = __float_as_uint(a.accumulate ? __uint_as_float(o[i]) + r[i] : r[i]);
            write_as<u32x4>(to, o);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (at + i < end) {
                    float* const to = at + i < size ? a.dw + at + i : a.db + (at + i - size);
                    *to = a.accumulate ? *to + r[i] : r[i];
                }
        }
    }
}

// ------------------------------------------------------------------------------------------------
// launches
// ------------------------------------------------------------------------------------------------
static int64_t part_stride(int64_t n, int64_t k) { return (n * k + n + 3) & ~int64_t(3); }
size_t ckpt_wgrad_workspace(int64_t rows, int64_t n, int64_t k)
{
    size_t most = FF_WS_MIN_BYTES;
    for (int terms = 1; terms <= 3; ++terms) {
        const WgradPlan p = wgrad_plan(rows, n, k, terms);
        const size_t need = p.splits > 1 ? align_up((size_t)p.splits * (size_t)part_stride(n, k) * sizeof(float), 256) : 0;
        if (need > most) most = need;
    }
    return most;
}

template <typename T> static hipError_t wgrad_of(const CkptWgradLaunch& l, hipStream_t s)
{
    const WgradPlan p = wgrad_plan(l.rows, l.n, l.k, Terms<T>::N);
    WgradArgs a;
    a.dy = l.dy;
    a.lddy = l.lddy;
    a.c = ckpt_ptr(l.q, l.e, l.k);
    a.rows = l.rows;
    a.n = (int32_t)l.n;
    a.k = (int32_t)l.k;
    a.tiles_n = (int32_t)((l.n + p.tile - 1) / p.tile);
    a.tiles_k = (int32_t)((l.k + p.tile - 1) / p.tile);
    a.splits = l.rows > 0 ? p.splits : 0;
    a.steps = p.steps;
    a.per = p.per;
    const int bm = plan_rows(Terms<T>::N, p.tile);
    const bool near = bm * l.lddy * (int64_t)sizeof(T) < int64_t(1) << 30;   // (offsets inside a step are 32 bits)
    a.plain = !near ? 0 : sizeof(T) == 2 && l.n % 2 != 0 ? p.steps - 1 : p.steps;
    a.gamma = l.gamma;
    a.beta = l.beta;
    a.param_kind = l.param_dtype;
    a.dw = l.dw;
    a.db = l.db;
    a.accumulate = l.accumulate;
    a.part = (float*)l.ws;
    a.stride = part_stride(l.n, l.k);
    if (l.rows > 0) {
        const unsigned grid = (unsigned)(((int64_t)a.tiles_n * a.tiles_k * a.splits + 7) / 8 * 8);
        if (p.tile == 256) k_ckpt_wgrad<T, 256, 4><<<grid, 512, 0, s>>>(a);
        else if (p.tile == 128) k_ckpt_wgrad<T, 128, 2><<<grid, 256, 0, s>>>(a);
        else k_ckpt_wgrad<T, 64, 2><<<grid, 256, 0, s>>>(a);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    if (a.splits != 1) {
        // (one round of the sum for all that is split; dw may have more elements than a launch has lanes for where there are no rows)
        const int64_t all = (int64_t)a.n * a.k + a.n, wgs = (all + 1023) / 1024, most = int64_t(1) << 20;
        k_ckpt_wgrad_sum<<<dim3((unsigned)(wgs < most ? wgs : most)), 256, 0, s>>>(a);
        return hipGetLastError();
    }
    return hipSuccess;
}
hipError_t launch_ckpt_wgrad(const CkptWgradLaunch& a, hipStream_t s)
{
    return a.dtype == FF_F32 ? wgrad_of<float>(a, s) : a.dtype == FF_BF16 ? wgrad_of<bf16_t>(a, s) : wgrad_of<f16_t>(a, s);
}

}  // namespace ffi
