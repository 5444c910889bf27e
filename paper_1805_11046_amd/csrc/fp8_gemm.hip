// Products of 8-bit floating point codes with a scale for each block of 128 of the reduction: out[m][n] = sum_k A[m][k] B[n][k].
//
// Two ways to multiply, by the type of the result:
//   bf16: the 8-bit matrix instruction over 128 entries, which takes the scales as operands, a byte (exponent + 127) for every row of
//     either operand: a block of 128 is one instruction and its scaling costs nothing.  Inside, it adds products in groups of eight
//     and there loses what lies below 2^-13 of the group's largest (measured: 1 + 2^-13 is kept, 1 + 2^-14 is 1; over random operands
//     the result is 0.8e-5 to 1.5e-5 off in the 2-norm), the sums of groups are fp32.  A bf16 result is off by up to 2^-8 anyway.
//   fp32: codes become bf16 values with their scale already on, two in an instruction and exactly (a code has at most four
//     significant bits, and what they stand for came out of a fp32 value), and the bf16 matrix instruction adds them in fp32
//     (2e-8 off).  Half the rate of the 8-bit one, which such results need: every fp8 instruction of this chip, with scales or
//     without, adds in the same groups.
// Both operands are read with one assignment of a lane's registers to positions inside a block; which it is does not matter to a
// sum over the block.  Rows are whole blocks (filled up with zeros), so the reduction has no tail; rows behind the last are read
// as the last one and not stored: a row of the result depends on its own row of A and its own row of B alone.
#include <type_traits>

#include "fp8_codes.h"

namespace {

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef q8t_bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef q8t_bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef q8t_bf16 bf16x8 __attribute__((ext_vector_type(8)));

// eight codes times the power of two s
template <int FMT>
__device__ __forceinline__ bf16x8 widen(int lo, int hi, float s)
{
    auto two = [&](int w, auto high) {
        constexpr bool H = decltype(high)::value;
        return FMT == Q8T_E4M3 ? (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, H)
                               : (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, s, H);
    };
    const bf16x2 a = two(lo, std::false_type()), b = two(lo, std::true_type()), c = two(hi, std::false_type()), d = two(hi, std::true_type());
    const bf16x4 ab = __builtin_shufflevector(a, b, 0, 1, 2, 3), cd = __builtin_shufflevector(c, d, 0, 1, 2, 3);
    return __builtin_shufflevector(ab, cd, 0, 1, 2, 3, 4, 5, 6, 7);
}

// One row's part of a block in a lane: a quarter of its 128 entries.  FMT: e4m3 or e5m2; WIDE: as bf16 values times their scale.
template <int FMT, bool WIDE>
struct Part;
template <int FMT>
struct Part<FMT, false> {
    i32x8 v;
    int scale;
    // lo, hi: 16 codes each; scales: those of four blocks, BYTE the one of this block
    template <int BYTE>
    __device__ __forceinline__ void set(i32x4 lo, i32x4 hi, int scales)
    {
        v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        scale = scales;
    }
};
template <int FMT>
struct Part<FMT, true> {
    bf16x8 v[4];
    template <int BYTE>
    __device__ __forceinline__ void set(i32x4 lo, i32x4 hi, int scales)
    {
        const float s = __uint_as_float((((uint32_t)scales >> (8 * BYTE)) & 255u) << 23);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = widen<FMT>(i < 2 ? lo[2 * i] : hi[2 * i - 4], i < 2 ? lo[2 * i + 1] : hi[2 * i - 3], s);
    }
};

// D[i][j] += sum over the block of P[i][.] Q[j][.]; lane l holds entries of rows l % 16 of both and D[4 * (l / 16) + 0..3][l % 16]
template <int BYTE, int FP, int FQ>
__device__ __forceinline__ f32x4 block_product(const Part<FP, false> &p, const Part<FQ, false> &q, f32x4 acc)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(p.v, q.v, acc, FP, FQ, BYTE, p.scale, BYTE, q.scale);
}
template <int BYTE, int FP, int FQ>
__device__ __forceinline__ f32x4 block_product(const Part<FP, true> &p, const Part<FQ, true> &q, f32x4 acc)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p.v[i], q.v[i], acc, 0, 0, 0);
    return acc;
}

struct Product {
    const uint8_t *a, *sa, *b, *sb;
    int M, N, nk;        // nk: blocks of the reduction
    int64_t ld, lds;     // bytes of a row of codes, of scales
    void *out;
};

// four results of one row next to each other
template <class OUT>
__device__ __forceinline__ void store4(OUT *out, int64_t at, const f32x4 v, int count)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < count) out[at + i] = (OUT)v[i];
}

// Operands straight from memory to registers; the W wavefronts of a workgroup share a tile of 16*MT x 16*NT results and take turns at
// the reduction, four blocks at a time, because four scales of a row are one word.
template <int FA, int FB, class OUT, int MT, int NT, int W>
__global__ __launch_bounds__(64 * W) void direct(const Product p)
{
    constexpr bool WIDE = std::is_same<OUT, float>::value;
    __shared__ f32x4 fold[W > 1 ? W : 1][MT * NT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, r = lane & 15, g = lane / 16;
    const int n0 = blockIdx.x * (16 * NT), m0 = blockIdx.y * (16 * MT);
    const uint8_t *pa[MT], *psa[MT], *pb[NT], *psb[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t row = min(m0 + 16 * i + r, p.M - 1);
        pa[i] = p.a + row * p.ld + g * 16;
        psa[i] = p.sa + row * p.lds;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int64_t row = min(n0 + 16 * j + r, p.N - 1);
        pb[j] = p.b + row * p.ld + g * 16;
        psb[j] = p.sb + row * p.lds;
    }
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    for (int k0 = wave * 4; k0 < p.nk; k0 += 4 * W) {
        int sa[MT], sb[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) sa[i] = *reinterpret_cast<const int *>(psa[i] + k0);
#pragma unroll
        for (int j = 0; j < NT; ++j) sb[j] = *reinterpret_cast<const int *>(psb[j] + k0);
        auto step = [&](auto byte) {
            constexpr int B = decltype(byte)::value;
            if (k0 + B >= p.nk) return;
            const int64_t at = (int64_t)(k0 + B) * 128;
            Part<FA, WIDE> a[MT];
            Part<FB, WIDE> b[NT];
#pragma unroll
            for (int i = 0; i < MT; ++i)
                a[i].template set<B>(*reinterpret_cast<const i32x4 *>(pa[i] + at), *reinterpret_cast<const i32x4 *>(pa[i] + at + 64), sa[i]);
#pragma unroll
            for (int j = 0; j < NT; ++j)
                b[j].template set<B>(*reinterpret_cast<const i32x4 *>(pb[j] + at), *reinterpret_cast<const i32x4 *>(pb[j] + at + 64), sb[j]);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = block_product<B>(b[j], a[i], acc[i][j]);
        };
        step(std::integral_constant<int, 0>());
        step(std::integral_constant<int, 1>());
        step(std::integral_constant<int, 2>());
        step(std::integral_constant<int, 3>());
    }
    if (W > 1) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) fold[wave][i * NT + j][lane] = acc[i][j];
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            if ((i * NT + j) % W != wave) continue;   // the tiles are dealt out to the wavefronts
            f32x4 v = acc[i][j];
            if (W > 1) {
                v = fold[0][i * NT + j][lane];
#pragma unroll
                for (int w = 1; w < W; ++w) v += fold[w][i * NT + j][lane];
            }
            const int m = m0 + 16 * i + r, n = n0 + 16 * j + 4 * g;
            if (m < p.M) store4((OUT *)p.out, (int64_t)m * p.N + n, v, p.N - n);
        }
}

template <int FA, int FB, class OUT>
int run(const Product &p, hipStream_t st)
{
    if (p.M <= 16) {
        direct<FA, FB, OUT, 1, 1, 8><<<dim3((p.N + 15) / 16, (p.M + 15) / 16), 512, 0, st>>>(p);
    } else {
        direct<FA, FB, OUT, 4, 4, 4><<<dim3((p.N + 63) / 64, (p.M + 63) / 64), 256, 0, st>>>(p);
    }
    Q8T_LAUNCH_CHECK();
    return Q8T_OK;
}
template <class OUT>
int by_format(const Product &p, int fa, int fb, hipStream_t st)
{
    if (fa == Q8T_E4M3) return fb == Q8T_E4M3 ? run<Q8T_E4M3, Q8T_E4M3, OUT>(p, st) : run<Q8T_E4M3, Q8T_E5M2, OUT>(p, st);
    return fb == Q8T_E4M3 ? run<Q8T_E5M2, Q8T_E4M3, OUT>(p, st) : run<Q8T_E5M2, Q8T_E5M2, OUT>(p, st);
}

}  // namespace

extern "C" {

size_t q8t_fp8_gemm_workspace_size(int M, int N, int K)
{
    (void)M, (void)N, (void)K;
    return 0;
}

int q8t_fp8_gemm(const uint8_t *a, const uint8_t *sa, int format_a, const uint8_t *b, const uint8_t *sb, int format_b, int M, int N, int K,
                 void *out, int type, void *ws, void *stream)
{
    if (M < 0 || N < 0 || K <= 0 || K > (1 << 30) || M > (1 << 22) || N > (1 << 22)) return Q8T_ERR_SHAPE;
    if ((type != Q8T_F32 && type != Q8T_BF16) || (format_a != Q8T_E4M3 && format_a != Q8T_E5M2) ||
        (format_b != Q8T_E4M3 && format_b != Q8T_E5M2))
        return Q8T_ERR_VALUE;
    if (M == 0 || N == 0) return Q8T_OK;
    if (!a || !sa || !b || !sb || !out) return Q8T_ERR_NULL;
    if (!q8t_aligned(a, 16) || !q8t_aligned(b, 16) || !q8t_aligned(sa, 4) || !q8t_aligned(sb, 4)) return Q8T_ERR_SHAPE;
    (void)ws;
    const Product p = {a, sa, b, sb, M, N, (K + 127) / 128, fp8_row_bytes(K), fp8_scale_bytes(K), out};
    return type == Q8T_F32 ? by_format<float>(p, format_a, format_b, (hipStream_t)stream)
                           : by_format<q8t_bf16>(p, format_a, format_b, (hipStream_t)stream);
}

}  // extern "C"
