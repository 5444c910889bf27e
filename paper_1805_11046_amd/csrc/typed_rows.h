// Tensors of fp32 or bf16 values, eight at a time: what the row kernels (residual_norm.hip, dropout.hip, fp8_quantize.hip)
// share.  All arithmetic is fp32; a bf16 result is rounded to nearest even once, where it is stored.
#pragma once
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

template <class T>
__device__ __forceinline__ float q8t_to_f32(T v)
{
    return (float)v;
}

// v[0..7] = p[0..7]; FULL: all there, else `count` (may be <= 0) of them and 0 for the others.  Streamed tensors are read past
// the caches (non-temporal), as everywhere in the library.
template <class T>
__device__ __forceinline__ void q8t_load8(const T *p, float v[8])
{
    typedef typename Q8tRaw<sizeof(T)>::type raw;
    constexpr int PER = 16 / sizeof(T);
#pragma unroll
    for (int h = 0; h < 8 / PER; ++h) {
        const raw w = __builtin_nontemporal_load(reinterpret_cast<const raw *>(p) + h);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (sizeof(T) == 4) v[h * PER + i] = __uint_as_float(w[i]);
            else v[h * PER + i] = __uint_as_float((i & 1) ? (w[i >> 1] & 0xFFFF0000u) : (w[i >> 1] << 16));
        }
    }
}
template <class T>
__device__ __forceinline__ void q8t_load8(const T *p, float v[8], int count)
{
    if (count >= 8) {
        q8t_load8(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < count ? q8t_to_f32(p[i]) : 0.0f;
}

// weights and gates: small, read again by every row, so through the caches
template <class T>
__device__ __forceinline__ void q8t_load8_kept(const T *p, float v[8], int count)
{
    typedef typename Q8tRaw<sizeof(T)>::type raw;
    constexpr int PER = 16 / sizeof(T);
    if (count >= 8) {
#pragma unroll
        for (int h = 0; h < 8 / PER; ++h) {
            const raw w = reinterpret_cast<const raw *>(p)[h];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (sizeof(T) == 4) v[h * PER + i] = __uint_as_float(w[i]);
                else v[h * PER + i] = __uint_as_float((i & 1) ? (w[i >> 1] & 0xFFFF0000u) : (w[i >> 1] << 16));
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < count ? q8t_to_f32(p[i]) : 0.0f;
}

__device__ __forceinline__ uint32_t q8t_pack_bf16(float a, float b)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef q8t_bf16 b2 __attribute__((ext_vector_type(2)));
    const f2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
}

template <class T>
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
        reinterpret_cast<raw *>(p)[h] = w;
    }
}
template <class T>
__device__ __forceinline__ void q8t_store8(T *p, const float v[8], int count)
{
    if (count >= 8) {
        q8t_store8(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < count) p[i] = (T)v[i];
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

// the generator's 16 bits for the 8 flat positions from i on; ALIGNED: i is a multiple of 4
template <bool ALIGNED>
__device__ __forceinline__ void q8t_draw8(int64_t i, const Q8tSeed &s, uint32_t r[8])
{
    uint32_t w[6];
    const uint32_t g = (uint32_t)(i >> 2);
    rng_group(g, s.lo, s.hi, w[0], w[1]);
    rng_group(g + 1, s.lo, s.hi, w[2], w[3]);
    if (ALIGNED) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            r[2 * k] = w[k] & 0xFFFFu;
            r[2 * k + 1] = w[k] >> 16;
        }
        return;
    }
    rng_group(g + 2, s.lo, s.hi, w[4], w[5]);
    const bool two = i & 2, one = i & 1;   // the window starts up to three halfwords into the three groups
    uint32_t v[5];
#pragma unroll
    for (int k = 0; k < 5; ++k) v[k] = two ? w[k + 1] : w[k];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t x = one ? (v[k] >> 16) | (v[k + 1] << 16) : v[k];
        r[2 * k] = x & 0xFFFFu;
        r[2 * k + 1] = x >> 16;
    }
}

// drop-out: position kept iff its 16 bits reach `cut`
struct Q8tDrop {
    uint32_t cut;
    float scale;   // 65536 / (65536 - cut); 0 where nothing is kept
};
static inline bool q8t_drop(double p, Q8tDrop *d)
{
    if (!(p >= 0.0 && p <= 1.0)) return false;
    d->cut = (uint32_t)__builtin_rint(p * 65536.0);
    d->scale = d->cut < 65536u ? (float)(65536.0 / (double)(65536u - d->cut)) : 0.0f;
    return true;
}
