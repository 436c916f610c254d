// Device code shared by the layer norm (norm.hip), the 8-bit checkpoints (ckpt.hip) and the weight gradient read from them
// (ckpt_wgrad.hip): rows of fp32 / bf16 / fp16 values in chunks of eight, and the checkpoint's codes.
//
// A checkpoint holds, for every 32 consecutive columns of a row (a block), int8 codes q and one exponent byte e: the value is
// q * 2^(e - 127).  The exponent s = e - 127 is the smallest integer with absmax <= 127 * 2^s, so that no code is ever clamped and
// stochastic rounding stays unbiased (it is capped at 121, where the largest fp32 values are; there the clamp holds the code at 127).  A power of
// two and not absmax / 127: scaling is exact, a value has seven significant bits and is exact in bf16, which is what lets the weight gradient
// multiply checkpoints in bf16 without rounding them again; the price is up to one bit of the code.  absmax below 2^-100: zero codes, e = 127, as in the
// per-tensor quantiser.  A block that holds an infinity or a NaN: zero codes and e = 255, and every value of it reads as NaN.
#pragma once

#include "device_math.hpp"
#include "ff_internal.hpp"

namespace ffi {

struct bf16_t { uint16_t b; };
struct f16_t { uint16_t b; };
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// Words at any address that is a multiple of the element's size: rows of odd length and views with any row stride take the same wide
// instructions as aligned ones (global memory instructions need no alignment here).
template <typename W, typename T> struct __attribute__((packed, aligned(sizeof(T)))) Packed { W v; };
template <typename W, typename T> __device__ __forceinline__ W read_as(const T* p) { return ((const Packed<W, T>*)p)->v; }
template <typename W, typename T> __device__ __forceinline__ void write_as(T* p, W v) { ((Packed<W, T>*)p)->v = v; }

__device__ __forceinline__ float bf16_value(uint32_t b) { return __uint_as_float(b << 16); }
// round to nearest even; NaN stays NaN
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    const v2bf p = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ uint32_t f16_pair(float lo, float hi)
{
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
    const v2h p = {(_Float16)lo, (_Float16)hi};
    return __builtin_bit_cast(uint32_t, p);
}

// Eight consecutive elements as they lie in memory.
template <typename T> struct Raw8;
template <> struct Raw8<float> { u32x4 a, b; };
template <> struct Raw8<bf16_t> { u32x4 a; };
template <> struct Raw8<f16_t> { u32x4 a; };

__device__ __forceinline__ void raw_zero(Raw8<float>& r) { r.a = r.b = u32x4{0, 0, 0, 0}; }
__device__ __forceinline__ void raw_zero(Raw8<bf16_t>& r) { r.a = u32x4{0, 0, 0, 0}; }
__device__ __forceinline__ void raw_zero(Raw8<f16_t>& r) { r.a = u32x4{0, 0, 0, 0}; }

// n elements (0 .. 8) at p; those beyond are zero.  Fewer than eight: four, two and one of them by n's bits.
template <typename T> __device__ __forceinline__ Raw8<T> load_raw(const T* p, int n)
{
    Raw8<T> r;
    raw_zero(r);
    const bool four = n & 4, two = n & 2, one = n & 1;
    if (n >= 8) {
        r.a = read_as<u32x4>(p);
        if constexpr (sizeof(T) == 4) r.b = read_as<u32x4>(p + 4);
    } else if constexpr (sizeof(T) == 4) {
        u32x4 f = {0, 0, 0, 0};
        u32x2 t = {0, 0};
        uint32_t o = 0;
        if (four) f = read_as<u32x4>(p);
        if (two) t = read_as<u32x2>(p + (n & 4));
        if (one) o = read_as<uint32_t>(p + (n & 6));
        const u32x4 rest = {two ? t[0] : o, t[1], two ? o : 0u, 0u};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            r.a[i] = four ? f[i] : rest[i];
            r.b[i] = four ? rest[i] : 0u;
        }
    } else {
        u32x2 f = {0, 0};
        uint32_t t = 0, o = 0;
        if (four) f = read_as<u32x2>(p);
        if (two) t = read_as<uint32_t>(p + (n & 4));
        if (one) o = read_as<uint16_t>(p + (n & 6));
        const uint32_t rest0 = two ? t : o, rest1 = two ? o : 0u;
        r.a = u32x4{four ? f[0] : rest0, four ? f[1] : rest1, four ? rest0 : 0u, four ? rest1 : 0u};
    }
    return r;
}
__device__ __forceinline__ void raw_values(const Raw8<float>& r, float v[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = __uint_as_float(r.a[i]);
        v[4 + i] = __uint_as_float(r.b[i]);
    }
}
__device__ __forceinline__ void raw_values(const Raw8<bf16_t>& r, float v[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(r.a[i] << 16);
        v[2 * i + 1] = __uint_as_float(r.a[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void raw_values(const Raw8<f16_t>& r, float v[8])
{
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const v2h p = __builtin_bit_cast(v2h, (uint32_t)r.a[i]);
        v[2 * i] = (float)p.x;
        v[2 * i + 1] = (float)p.y;
    }
}
__device__ __forceinline__ void raw_of(const float v[8], Raw8<float>& r)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.a[i] = __float_as_uint(v[i]);
        r.b[i] = __float_as_uint(v[4 + i]);
    }
}
__device__ __forceinline__ void raw_of(const float v[8], Raw8<bf16_t>& r)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) r.a[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
}
__device__ __forceinline__ void raw_of(const float v[8], Raw8<f16_t>& r)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) r.a[i] = f16_pair(v[2 * i], v[2 * i + 1]);
}
template <typename T> __device__ __forceinline__ void store_raw(T* p, int n, const Raw8<T>& r)
{
    const bool four = n & 4, two = n & 2, one = n & 1;
    if (n >= 8) {
        write_as<u32x4>(p, r.a);
        if constexpr (sizeof(T) == 4) write_as<u32x4>(p + 4, r.b);
    } else if constexpr (sizeof(T) == 4) {
        const u32x4 rest = four ? r.b : r.a;
        if (four) write_as<u32x4>(p, r.a);
        if (two) write_as<u32x2>(p + (n & 4), u32x2{rest[0], rest[1]});
        if (one) write_as<uint32_t>(p + (n & 6), two ? rest[2] : rest[0]);
    } else {
        const uint32_t rest0 = four ? r.a[2] : r.a[0], rest1 = four ? r.a[3] : r.a[1];
        if (four) write_as<u32x2>(p, u32x2{r.a[0], r.a[1]});
        if (two) write_as<uint32_t>(p + (n & 4), rest0);
        if (one) write_as<uint16_t>(p + (n & 6), (uint16_t)(two ? rest1 : rest0));
    }
}
template <typename T> __device__ __forceinline__ void load8(const T* p, int n, float v[8])
{
    const Raw8<T> r = load_raw(p, n);
    raw_values(r, v);
}
template <typename T> __device__ __forceinline__ void store8(T* p, int n, const float v[8])
{
    Raw8<T> r;
    raw_of(v, r);
    store_raw(p, n, r);
}

// Values that the compiler is not to trace back.  It would keep what it made of them before instead of making it again, which takes more registers
// than there are, or take them apart right behind the load, which waits for it there.
__device__ __forceinline__ void opaque(u32x4& v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void opaque(u32x2& v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void opaque(Raw8<float>& r) { opaque(r.a); opaque(r.b); }
__device__ __forceinline__ void opaque(Raw8<bf16_t>& r) { opaque(r.a); }
__device__ __forceinline__ void opaque(Raw8<f16_t>& r) { opaque(r.a); }
__device__ __forceinline__ void opaque(uint32_t& v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void opaque_uniform(int& v) { asm volatile("" : "+s"(v)); }
__device__ __forceinline__ void opaque(float& v) { asm volatile("" : "+v"(v)); }

// Element `at` of row row0 + r: row0, the workgroup's part, is scalar, a lane's is one product of 32 by 32 bits (rows are at most 2^31 elements apart).
template <typename T> __device__ __forceinline__ T* element(T* p, int64_t ld, int64_t row0, uint32_t r, uint32_t at)
{
    return p + row0 * ld + ((uint64_t)r * (uint32_t)ld + at);
}

// ---- a row's chunks -----------------------------------------------------------------------------------------------------
// Where rows end: with a chunk; inside one, with at least eight columns; anywhere; anywhere, and no column but the chunk's own is read, because other
// lanes may write theirs first.
enum RowEnds { ROWS_WHOLE, ROWS_RAGGED, ROWS_ANY, ROWS_OWN };
// Chunk c, n of whose columns exist (none: n <= 0), without a branch, behind which the compiler would count on fewer loads under way than there are.
// What is not there is read from the row's first chunk, and the chunk that a row ends in as the row's last eight columns; `settle` makes zeros of what does
// not exist when the values are needed.
template <RowEnds ENDS, typename T> __device__ __forceinline__ Raw8<T> row_chunk(const T* row, int c, int n, int cols)
{
    if (ENDS == ROWS_OWN || (ENDS == ROWS_ANY && cols < 8)) return load_raw(row + 8 * c, max(0, n));
    return load_raw(row + (n <= 0 ? 0 : ENDS != ROWS_WHOLE && n < 8 ? cols - 8 : 8 * c), 8);
}
template <int WORD> __device__ __forceinline__ void move_down(uint32_t (&w)[8 / WORD], int by)   // by: elements, 1 .. 8; WORD: elements of a word
{
    constexpr int W = 8 / WORD;
#pragma unroll
    for (int step = 4; step >= WORD; step /= 2)
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = by & step ? (i + step / WORD < W ? w[i + step / WORD] : 0u) : w[i];
    if constexpr (WORD == 2)
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = by & 1 ? __builtin_amdgcn_alignbit(i + 1 < W ? w[i + 1] : 0u, w[i], 16) : w[i];
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = by & 8 ? 0u : w[i];
}
template <RowEnds ENDS, typename T> __device__ __forceinline__ void settle(Raw8<T>& r, int n, int cols)
{
    if (n >= 8 || ENDS == ROWS_OWN || (ENDS == ROWS_ANY && cols < 8)) return;
    constexpr int W = sizeof(T) == 4 ? 8 : 4;
    uint32_t w[W];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = r.a[i];
        if constexpr (W == 8) w[4 + i] = r.b[i];
    }
    if constexpr (ENDS != ROWS_WHOLE) {
        move_down<8 / W>(w, 8 - max(0, n));
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = 0;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.a[i] = w[i];
        if constexpr (W == 8) r.b[i] = w[4 + i];
    }
}

// ---- a block's exponent byte and the codes of a chunk -------------------------------------------------------------------
// A chunk is a lane's eight columns; the four lanes of a quad hold a block.
__device__ __forceinline__ uint32_t quad_max_u32(uint32_t v)
{
    v = max(v, dpp_u32<0xB1>(v));   // quad_perm [1,0,3,2]
    v = max(v, dpp_u32<0x4E>(v));   // quad_perm [2,3,0,1]
    return v;
}
__device__ __forceinline__ uint32_t abs_max_bits(const float v[8])
{
    // bits have the order of the sizes: among values without a sign as signed integers, and among those with one as unsigned, above all others
    int32_t p = 0;
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        p = max(p, __float_as_int(v[i]));
        n = max(n, __float_as_uint(v[i]));
    }
    return max((uint32_t)p, n & 0x7FFFFFFFu);
}
// absmax = m * 2^E, 1 <= m < 2: s = E - 6, one more where m > 127/64, which is where adding 0x1FFFF carries into the exponent
__device__ __forceinline__ uint32_t ckpt_exponent(uint32_t amax_bits)
{
    const uint32_t e = min(((amax_bits + 0x1FFFFu) >> 23) - 6u, 248u);
    return amax_bits >= 0x7F800000u ? 255u : (amax_bits < (27u << 23) ? 127u : e);
}
__device__ __forceinline__ float ckpt_scale(uint32_t e) { return __uint_as_float(e << 23); }   // e = 255: infinity, and 0 * it NaN

// sr_head of elements at .. at + 7; FOURS: at is a multiple of four
template <bool FOURS = false> __device__ __forceinline__ void sr_words8(const SrKey& key, uint64_t at, uint32_t w[8])
{
    const uint32_t lo = (uint32_t)at, k = key.k0 + (uint32_t)(at >> 32) * key.k1;
    if (FOURS || (lo & 3u) == 0) {
        sr_head4(lo ^ k, w);
        sr_head4((lo + 4u) ^ (lo + 4u < lo ? k + key.k1 : k), w + 4);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = sr_head((lo + i) ^ (lo + i < lo ? k + key.k1 : k));
    }
}

struct CkptRound {   // how codes are rounded; filled in by the launch
    SrKey key;
    int32_t stochastic;
};
// at: row-major element index of the chunk's first column (FOURS: a multiple of four)
template <bool FOURS = false> __device__ __forceinline__ u32x2 ckpt_codes(const float v[8], uint32_t amax_bits, uint32_t e, const CkptRound& c, uint64_t at)
{
    const uint32_t some = amax_bits >= (27u << 23) && amax_bits < 0x7F800000u ? 0xFFFFFFFFu : 0u;
    const float inv = __uint_as_float((254u - e) << 23);   // (not used where e is 127 or 255 for another reason)
    u32x2 q;
    if (c.stochastic) {
        uint32_t w[8];
        sr_words8<FOURS>(c.key, at, w);
        // what sr_scale makes of t = v * inv, of t 2^24 = v 2^p: one product less
        const int p = 151 - (int)e;
        uint32_t x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float t = -__builtin_amdgcn_ldexpf(v[i], p), one = __builtin_amdgcn_fmed3f(t * 0x1p127f, 0.0f, 1.0f);
            x[i] = sr_top(__builtin_fmaf(one, 0x1p24f, __builtin_fmaf(one, -0x1p24f, t)), -SR_MOST, SR_MOST, w[i]);
        }
        q[0] = sr_pack(x[0], x[1], x[2], x[3]);
        q[1] = sr_pack(x[4], x[5], x[6], x[7]);
    } else {
        // 1.5 * 2^23 + t: the sum's last place is one, and its low byte the code
        uint32_t x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __float_as_uint(__builtin_amdgcn_fmed3f(v[i] * inv, -127.0f, 127.0f) + 12582912.0f);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t a = __builtin_amdgcn_perm(x[4 * h + 1], x[4 * h], 0x0C0C0400u);
            const uint32_t b = __builtin_amdgcn_perm(x[4 * h + 3], x[4 * h + 2], 0x04000C0Cu);
            q[h] = a | b;
        }
    }
    return q & some;
}
__device__ __forceinline__ void ckpt_values(u32x2 q, uint32_t e, float v[8])
{
    const float s = ckpt_scale(e);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(int8_t)(q[i >> 2] >> (8 * (i & 3))) * s;
}

// ---- launch arguments ------------------------------------------------------------------------------------------------
// One matrix of a checkpoint: codes with their row pitch, exponent bytes with theirs.
struct CkptPtr {
    int8_t* q;
    uint8_t* e;
    int64_t pitch;    // of q: ff_pitch(cols)
    int64_t epitch;   // of e: ff_pitch(blocks)
    int32_t blocks;
};
static inline int64_t ckpt_blocks(int64_t cols) { return (cols + FF_CKPT_BLOCK - 1) / FF_CKPT_BLOCK; }
static inline CkptPtr ckpt_ptr(const void* q, const void* e, int64_t cols)
{
    const int64_t nb = ckpt_blocks(cols);
    return {(int8_t*)q, (uint8_t*)e, pitch8(cols), pitch8(nb), (int32_t)nb};
}
// Lane `chunk` of a row's `slots` lanes (a multiple of four that covers the row's pitch) stores its chunk's codes, its block's exponent and its share of
// the pad bytes, which are zero.  `live`: the lane's chunk holds columns; q_row, e_row: where the row begins.
__device__ __forceinline__ void ckpt_store_chunk(const CkptPtr& k, int8_t* q_row, uint8_t* e_row, int chunk, int slots, bool live, u32x2 q, uint32_t e)
{
    if ((int64_t)chunk * 8 < k.pitch) *(u32x2*)(q_row + (uint32_t)chunk * 8) = live ? q : u32x2{0, 0};
    const int b = chunk >> 2;
    if ((chunk & 3) == 0 && b < k.blocks) e_row[b] = (uint8_t)e;
    for (int p = k.blocks + chunk; p < (int)k.epitch; p += slots) e_row[p] = 0;
}

}  // namespace ffi
