// Dropout whose mask is never stored: y = r + (u >= p ? x / (1 - p) : 0), u the uniform of the element's random word.  The backward pass is the same
// call on the gradient: the words depend on (seed, tag, element) alone.
//
// Bound by memory.  The word is the quantiser's (device_math.hpp), about ten operations a value, and its comparison takes the word
// as it is: u = (word >> 8) 2^-24 >= p where word >= ceil(p 2^24) 2^8.  Two chunks of eight values a thread, loaded before either is used.
// Measured: 16384 x 4096 bf16 with a residual 70 us (5.7 TB/s, 20 vector instructions a value); 64 x 500 fp32 3.9 us, the launch.
#include "chunks.hpp"
#include "blocks.hpp"

namespace ffi {

template <typename T> struct DropoutArgs {
    Chunks c;
    const T* x;
    const T* r;        // may be null
    T* y;
    int64_t ldx, ldr, ldy;
    uint64_t seed, tag;
    const uint64_t* step_dev;   // may be null
    float scale;
    uint32_t least;    // the smallest word that keeps its element
    int32_t none;      // no element is kept
    int32_t cols;
};

template <typename T, RowEnds ENDS, bool RESIDUAL, int U> __global__ __launch_bounds__(CK_THREADS) void k_dropout(DropoutArgs<T> a)
{
    const int64_t first = (int64_t)blockIdx.x * (CK_THREADS * U);
    int64_t row0;
    uint32_t chunk0;
    chunk_first(a.c, first, row0, chunk0);
    Raw8<T> x[U], res[RESIDUAL ? U : 1];
    uint32_t r[U], chunk[U];
    int n[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        n[i] = chunk_at(a.c, a.cols, first, chunk0, i * CK_THREADS + threadIdx.x, r[i], chunk[i]);
        x[i] = row_chunk<ENDS>(element(a.x, a.ldx, row0, r[i], 0), (int)chunk[i], n[i], a.cols);
        if constexpr (RESIDUAL) res[i] = row_chunk<ENDS>(element(a.r, a.ldr, row0, r[i], 0), (int)chunk[i], n[i], a.cols);
    }
    const SrKey key = make_sr_key(a.seed, a.tag + (a.step_dev ? a.step_dev[0] << 20 : 0));
#pragma unroll
    for (int i = 0; i < U; ++i) {
        float v[8], w[8];
        settle<ENDS>(x[i], n[i], a.cols);
        raw_values(x[i], v);
        if constexpr (RESIDUAL) {
            settle<ENDS>(res[i], n[i], a.cols);
            raw_values(res[i], w);
        }
        uint32_t word[8];
        sr_words8(key, (uint64_t)row0 * (uint64_t)a.cols + ((uint64_t)r[i] * (uint32_t)a.cols + 8 * chunk[i]), word);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t h = word[j] ^ (word[j] >> 16);
            v[j] = h >= a.least && !a.none ? v[j] * a.scale : 0.0f;
            if constexpr (RESIDUAL) v[j] += w[j];
        }
        if (n[i] > 0) store8(element(a.y, a.ldy, row0, r[i], 8 * chunk[i]), n[i], v);
    }
}

template <typename T> static hipError_t dropout_of(const DropoutLaunch& d, hipStream_t s)
{
    DropoutArgs<T> a = {};
    a.c = chunks_of(d.rows, d.cols);
    a.x = (const T*)d.x;
    a.r = (const T*)d.r;
    a.y = (T*)d.y;
    a.ldx = d.ldx;
    a.ldr = d.ldr;
    a.ldy = d.ldy;
    a.seed = d.seed;
    a.tag = d.tag;
    a.step_dev = d.step_dev;
    a.cols = (int32_t)d.cols;
    const uint64_t least = (uint64_t)__builtin_ceil((double)d.p * 0x1p24) << 8;   // (p 2^24 is exact)
    a.none = least >> 32 != 0;
    a.least = (uint32_t)least;
    a.scale = a.none ? 0.0f : (float)(1.0 / (1.0 - (double)d.p));
    const unsigned grid = ckpt_grid<2>(a.c);
    by_ends(d.cols, d.x == d.y || d.r == d.y, [&](auto ends) {
        constexpr RowEnds E = decltype(ends)::value;
        if (a.r) k_dropout<T, E, true, 2><<<grid, CK_THREADS, 0, s>>>(a);
        else k_dropout<T, E, false, 2><<<grid, CK_THREADS, 0, s>>>(a);
    });
    return hipGetLastError();
}
hipError_t launch_dropout(const DropoutLaunch& d, hipStream_t s)
{
    return d.dtype == FF_F32 ? dropout_of<float>(d, s) : d.dtype == FF_BF16 ? dropout_of<bf16_t>(d, s) : dropout_of<f16_t>(d, s);
}

}  // namespace ffi
