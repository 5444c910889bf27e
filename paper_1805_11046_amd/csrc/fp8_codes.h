// 8-bit floating point codes with a power-of-two scale for each block of 128 (fp8_quantize.hip, residual_norm.hip).
//   e4m3: largest 448 = 1.75 * 2^8,   smallest normal 2^-6,  3 mantissa bits, NaN but no infinity
//   e5m2: largest 57344 = 1.75 * 2^15, smallest normal 2^-14, 2 mantissa bits, infinities and NaN
// Scale of a block: the smallest 2^E that brings its largest finite magnitude to at most 1.75 * 2^emax, so nothing saturates;
// stored as E + 127 in one byte, which the matrix instructions take as it is.  Division by a power of two is exact: a code
// carries one rounding and no more.
#pragma once
#include "typed_rows.h"

template <int FMT>
struct Fp8Format {
    static constexpr int EMAX = FMT == Q8T_E4M3 ? 8 : 15, EMIN = FMT == Q8T_E4M3 ? -6 : -14, MAN = FMT == Q8T_E4M3 ? 3 : 2;
};

static inline __host__ __device__ int64_t fp8_row_bytes(int64_t cols) { return (cols + 127) / 128 * 128; }
static inline __host__ __device__ int64_t fp8_scale_bytes(int64_t cols) { return ((cols + 127) / 128 + 3) / 4 * 4; }

// magnitude bits of a finite value, 0 for infinities and NaN: as whole numbers they are ordered like the magnitudes
__device__ __forceinline__ uint32_t fp8_magnitude(float x)
{
    const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
    return u < 0x7F800000u ? u : 0u;
}

// stored scale of a block with largest magnitude `u` (bits)
template <int FMT>
__device__ __forceinline__ uint32_t fp8_scale(uint32_t u)
{
    const int e = (int)(u >> 23) - Fp8Format<FMT>::EMAX + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);   // + 127 is in the field already
    return u == 0u ? 127u : (uint32_t)(e > 0 ? e : 0);
}
// 2^-E for the stored scale
__device__ __forceinline__ float fp8_inverse(uint32_t scale) { return __uint_as_float((254u - scale) << 23); }

// two scaled values, nearest even, in the low or high half of `old`
template <int FMT, bool HIGH>
__device__ __forceinline__ uint32_t fp8_pack2(float a, float b, uint32_t old)
{
    return (uint32_t)(FMT == Q8T_E4M3 ? __builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)old, HIGH)
                                      : __builtin_amdgcn_cvt_pk_bf8_f32(a, b, (int)old, HIGH));
}

// Stochastic codes.  With u = |v| / scale in steps of the code's last place, k = floor(u) + [frac(u) * 65536 > r + 0.5] for 16 bits r,
// in whole numbers.  c = 65535 - r.
//   normal codes: of the magnitude's bits m, SHIFT = 23 - MAN mantissa bits f go, and the condition is f >= (r << SHIFT - 16) +
//     2^(SHIFT - 17) + 1: adding 2^SHIFT less that, (c << SHIFT - 16) + 2^(SHIFT - 17) - 1, carries into what stays, up to the exponent.
//   below them all steps are of one size: |v| + least, `least` the smallest magnitude with a normal code, has the mantissa that the sum
//     above wants and an exponent one too high.  That sum has to be rounded up, so that a fraction just over the border stays over it.
// The larger of m and the second is the right one on both sides of `least`.  Needs fp8_round_up, and least >= 2^-126, that is scales
// above -EMIN; under others the values are scaled first (fp8_drawn), which is exact where the code is not 0.
template <int FMT>
struct Fp8Draw {
    typedef Fp8Format<FMT> F;
    static constexpr int SHIFT = 23 - F::MAN;
    uint32_t least;
    __device__ __forceinline__ explicit Fp8Draw(uint32_t scale) : least((uint32_t)((int)scale + F::EMIN) << 23) {}   // stored scale
    // 16 bits where they are added
    static __device__ __forceinline__ uint32_t drawn(uint32_t r16) { return ((65535u - r16) << (SHIFT - 16)) + (1u << (SHIFT - 17)) - 1u; }
    __device__ __forceinline__ uint32_t code(uint32_t m, uint32_t drawn) const
    {
        const uint32_t low = __float_as_uint(__uint_as_float(m) + __uint_as_float(least));
        return (max(m + 0x800000u, low) + drawn - least) >> SHIFT;
    }
};
// From here on additions in fp32 are rounded up in this wavefront, those of anything that is computed from the words given among them.
template <int N>
__device__ __forceinline__ void fp8_round_up(uint32_t (&first)[N])
{
    asm volatile("s_setreg_imm32_b32 hwreg(HW_REG_MODE, 0, 2), 1\n\ts_nop 3" : "+v"(first[0]));
#pragma unroll
    for (int i = 1; i < N; ++i) asm volatile("" : "+v"(first[i]));
}
// The code of any value v under any scale, given its inverse.
template <int FMT>
__device__ __forceinline__ uint32_t fp8_drawn(float v, float inverse, uint32_t drawn)
{
    const uint32_t b = __float_as_uint(v * inverse), m = b & 0x7FFFFFFFu, sign = b >> 24 & 0x80u;
    const uint32_t special = FMT == Q8T_E4M3 || m > 0x7F800000u ? 0x7Fu : 0x7Cu;
    return sign | (m >= 0x7F800000u ? special : Fp8Draw<FMT>(127u).code(m, drawn));
}

// 8 codes of values v under the stored scale (STOCH: behind fp8_round_up)
template <int FMT, bool STOCH>
__device__ __forceinline__ uint2 fp8_codes8(const float v[8], uint32_t scale, const uint32_t r[4])
{
    const float inv = fp8_inverse(scale);
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float *p = v + 4 * h;
        if (!STOCH) {
            w[h] = fp8_pack2<FMT, false>(p[0] * inv, p[1] * inv, 0u);
            w[h] = fp8_pack2<FMT, true>(p[2] * inv, p[3] * inv, w[h]);
        } else {
            w[h] = 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[h] |= fp8_drawn<FMT>(p[i], inv, Fp8Draw<FMT>::drawn(q8t_draw(r, 4 * h + i))) << (8 * i);
        }
    }
    return make_uint2(w[0], w[1]);
}

__device__ __forceinline__ uint32_t fp8_max8(const float v[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, fp8_magnitude(v[i]));
    return m;
}
// op over 16 consecutive lanes (one block of 128 at eight entries a lane); every one has the result
template <class Op>
__device__ __forceinline__ uint32_t fp8_fold16(uint32_t m, Op op)
{
    m = op(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));    // lanes 1 apart
    m = op(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));    // 2 apart
    m = op(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xF, 0xF, true));   // the other four of eight
    return op(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x140, 0xF, 0xF, true));   // the other eight
}
__device__ __forceinline__ uint32_t fp8_max16(uint32_t m)
{
    return fp8_fold16(m, [](uint32_t a, uint32_t b) { return max(a, b); });
}
