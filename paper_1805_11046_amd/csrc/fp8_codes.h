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

// stochastic code of a scaled value: k = floor(u) + [frac(u) * 65536 > r + 0.5] with u = |t| in steps of the code's last place
template <int FMT>
__device__ __forceinline__ uint32_t fp8_stochastic(float t, uint32_t r16)
{
    typedef Fp8Format<FMT> F;
    const uint32_t b = __float_as_uint(t), m = b & 0x7FFFFFFFu, sign = (b >> 24) & 0x80u;
    const uint32_t field = max(m >> 23, (uint32_t)(F::EMIN + 127));
    const float u = __uint_as_float(m) * __uint_as_float((254u + F::MAN - field) << 23);
    const float f = __builtin_floorf(u);
    const uint32_t k = (uint32_t)(int)f + ((u - f) * 65536.0f > (float)r16 + 0.5f ? 1u : 0u);
    const uint32_t code = ((field - (uint32_t)(F::EMIN + 127)) << F::MAN) + k;
    const uint32_t special = FMT == Q8T_E4M3 ? 0x7Fu : (m > 0x7F800000u ? 0x7Fu : 0x7Cu);
    return sign | (m >= 0x7F800000u ? special : code);
}

// 8 codes of values v under the stored scale
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
            for (int i = 0; i < 4; ++i) w[h] |= fp8_stochastic<FMT>(p[i] * inv, q8t_draw(r, 4 * h + i)) << (8 * i);
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
// over 16 consecutive lanes (one block of 128 at eight entries a lane)
__device__ __forceinline__ uint32_t fp8_max16(uint32_t m)
{
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off, 64));
    return m;
}
