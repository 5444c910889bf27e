// Tensors of fp32 or bf16 values, eight at a time: what the row kernels (residual_norm.hip, dropout.hip, fp8_quantize.hip)
// share.  All arithmetic is fp32; a bf16 result is rounded to nearest even once, where it is stored.
#pragma once
#include <type_traits>

#include "q8t_common.h"

typedef __bf16 q8t_bf16;

// 16 bytes at an address that need only be aligned as one element is: the memory pipeline takes a dwordx4 at any address
// (rows of an odd width start anywhere), so one form serves every width and view.
template <int BYTES>
struct Q8tRaw;
template <>
struct Q8tRaw<4> {
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4)));
};
template <>
struct Q8tRaw<2> {
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2)));
};

// entry c of a row by a byte offset that is a 32-bit number to the compiler as well: with a uniform row it is no address of 64 bits a lane
template <class T>
__device__ __forceinline__ T *q8t_at(T *row, uint32_t c)
{
    return reinterpret_cast<T *>(reinterpret_cast<uintptr_t>(row) + (uint32_t)(c * (uint32_t)sizeof(T)));
}

// Eight values as they lie in memory: what a kernel holds of a row it has asked for ahead.  Streamed tensors are read past the caches
// (non-temporal), as everywhere in the library; what every row reads again (weights, gates) comes through them.
template <class T>
struct Q8tEight {
    static constexpr int PER = 16 / sizeof(T), WORDS = 8 / PER * 4;
    uint32_t w[WORDS];
    template <bool STREAMED>
    __device__ __forceinline__ void vector(const T *p)
    {
        typedef typename Q8tRaw<sizeof(T)>::type raw;
#pragma unroll
        for (int h = 0; h < WORDS / 4; ++h) {
            const raw r = STREAMED ? __builtin_nontemporal_load(reinterpret_cast<const raw *>(p) + h) : reinterpret_cast<const raw *>(p)[h];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[4 * h + i] = r[i];
        }
    }
    // p[0 .. count - 1] one after the other, 0 behind them
    __device__ __forceinline__ void few(const T *p, int count)
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0u;
#pragma clang loop unroll(disable)
        for (int i = 0; i < count; ++i) {
            const uint32_t v = __float_as_uint((float)p[i]);
#pragma unroll
            for (int k = 0; k < WORDS; ++k) {
                if (sizeof(T) == 4) w[k] |= i == k ? v : 0u;
                else w[k] |= i >> 1 == k ? ((i & 1) ? v : v >> 16) : 0u;
            }
        }
    }
    // Asks for the entries c .. c + 7 of a row of D (`row` uniform in the wavefront: the address is a scalar and a 32-bit offset).  Where the
    // row has fewer behind c, its last eight are read in their place: no branch, and nothing waits here for them.  settle() puts them
    // right before they are used.  TINY: the row has fewer than eight entries in all.
    template <bool TINY, bool STREAMED = true>
    __device__ __forceinline__ void ask(const T *row, uint32_t c, uint32_t D)
    {
        if (TINY) few(row + min(c, D), (int)D - (int)c);
        else vector<STREAMED>(q8t_at(row, min(c, D - 8)));
    }
    template <bool TINY>
    __device__ __forceinline__ void settle(uint32_t c, uint32_t D)
    {
        if (TINY || c + 8 <= D) return;
        const uint32_t s = min(c + 8 - D, 8u);   // entries to drop in front; zeros follow behind (masks: see q8t_draw8)
        const int step = sizeof(T) == 4 ? 1 : 2;
#pragma unroll
        for (int d = 8; d >= step; d >>= 1) {
            const uint32_t on = (s & d) ? ~0u : 0u;
#pragma unroll
            for (int i = 0; i < WORDS; ++i) w[i] = (w[i] & ~on) | (i + d / step < WORDS ? w[i + d / step] & on : 0u);
        }
        if (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) w[i] = __builtin_amdgcn_alignbit(i + 1 < WORDS ? w[i + 1] : 0u, w[i], (s & 1) * 16);
        }
    }
    // What has been taken out of the words so far is taken out again after this: two values stay in one register in the meantime.
    __device__ __forceinline__ void hold()
    {
        if (sizeof(T) == 4) return;
#pragma unroll
        for (int i = 0; i < WORDS; ++i) asm volatile("" : "+v"(w[i]));
    }
    __device__ __forceinline__ uint32_t bits(int i) const   // of the value in fp32
    {
        if (sizeof(T) == 4) return w[i];
        return (i & 1) ? (w[i >> 1] & 0xFFFF0000u) : (w[i >> 1] << 16);
    }
    __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(bits(i)); }
};
// entries c .. c + 7 of a row through the caches, at once
template <bool TINY, class T>
__device__ __forceinline__ void q8t_row8(const T *row, float v[8], uint32_t c, uint32_t D)
{
    Q8tEight<T> e;
    e.template ask<TINY, false>(row, c, D);
    e.template settle<TINY>(c, D);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = e[i];
}
// p[0 .. count - 1] of a flat tensor
template <class T, bool STREAMED = true>
__device__ __forceinline__ void q8t_load8(const T *p, float v[8], int count)
{
    Q8tEight<T> e;
    if (count >= 8) e.template vector<STREAMED>(p);
    else e.few(p, count);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = e[i];
}

__device__ __forceinline__ uint32_t q8t_pack_bf16(float a, float b)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef q8t_bf16 b2 __attribute__((ext_vector_type(2)));
    const f2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
}

// STREAMED: past the caches, for results that nothing reads soon (forward pass of the norms over 8192 x 4096 bf16: 63.1 to 60.5 us)
template <bool STREAMED, class T>
__device__ __forceinline__ void q8t_store8(T *p, const float v[8])
{
    typedef typename Q8tRaw<sizeof(T)>::type raw;
    constexpr int PER = 16 / sizeof(T);
#pragma unroll
    for (int h = 0; h < 8 / PER; ++h) {
        raw w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (sizeof(T) == 4) w[i] = __float_as_uint(v[h * PER + i]);
            else w[i] = q8t_pack_bf16(v[2 * i], v[2 * i + 1]);
        }
        if (STREAMED) __builtin_nontemporal_store(w, reinterpret_cast<raw *>(p) + h);
        else reinterpret_cast<raw *>(p)[h] = w;
    }
}
template <bool STREAMED = false, class T>
__device__ __forceinline__ void q8t_store8(T *p, const float v[8], int count)
{
    if (count >= 8) {
        q8t_store8<STREAMED>(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < count) p[i] = (T)v[i];
}

// entries c .. c + 7 of a row of D (uniform in the wavefront)
template <bool STREAMED = false, class T>
__device__ __forceinline__ void q8t_row_store8(T *row, uint32_t c, const float v[8], uint32_t D)
{
    q8t_store8<STREAMED>(q8t_at(row, c), v, (int)D - (int)c);
}

// seed of a call: the host's plus the device counter, if there is one (a captured graph draws anew at every replay)
struct Q8tSeed {
    uint32_t lo, hi;
};
__device__ __forceinline__ Q8tSeed q8t_seed(uint64_t seed, const int64_t *step)
{
    const uint64_t s = seed + (step ? (uint64_t)*step : 0u);
    return {(uint32_t)s, (uint32_t)(s >> 32)};
}

// The generator's 16 bits for the 8 flat positions from i on, two in a word in their order.  ALIGNED: i is a multiple of 4.
template <bool ALIGNED>
__device__ __forceinline__ void q8t_draw8(int64_t i, const Q8tSeed &s, uint32_t r[4])
{
    uint32_t w[6];
    const uint32_t g = (uint32_t)(i >> 2);
    rng_group(g, s.lo, s.hi, w[0], w[1]);
    rng_group(g + 1, s.lo, s.hi, w[2], w[3]);
    if (ALIGNED) {
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] = w[k];
        return;
    }
    rng_group(g + 2, s.lo, s.hi, w[4], w[5]);
    // the window starts up to three halfwords into the three groups (masks, not choices: a choice between array entries is made by
    // address and would move the words to memory)
    const uint32_t two = (i & 2) ? ~0u : 0u, shift = (uint32_t)(i & 1) * 16;
    uint32_t v[5];
#pragma unroll
    for (int k = 0; k < 5; ++k) v[k] = (w[k] & ~two) | (w[k + 1] & two);
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = __builtin_amdgcn_alignbit(v[k + 1], v[k], shift);
}
__device__ __forceinline__ uint32_t q8t_draw(const uint32_t r[4], int k) { return (k & 1) ? r[k >> 1] >> 16 : r[k >> 1] & 0xFFFFu; }

// Drop-out: a position is kept iff its 16 bits reach `cut`.  `below` = (cut << 16) - 1 decides on a whole word, whose upper half the
// bits are: what is under them does not matter.
struct Q8tDrop {
    uint32_t cut, below;
    float scale;   // 65536 / (65536 - cut); 0 where nothing is kept
};
static inline bool q8t_drop(double p, Q8tDrop *d)
{
    if (!(p >= 0.0 && p <= 1.0)) return false;
    d->cut = (uint32_t)__builtin_rint(p * 65536.0);
    d->below = (d->cut << 16) - 1u;   // nothing is kept: all ones (and with cut = 0, where everything is, it is not asked)
    d->scale = d->cut < 65536u ? (float)(65536.0 / (double)(65536u - d->cut)) : 0.0f;
    return true;
}
__device__ __forceinline__ bool q8t_kept(const uint32_t r[4], int k, uint32_t below)
{
    return ((k & 1) ? r[k >> 1] : r[k >> 1] << 16) > below;
}
