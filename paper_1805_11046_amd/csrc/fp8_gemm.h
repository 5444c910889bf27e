// Products of 8-bit floating point codes with a scale for each block of 128 of the reduction: out[m][n] = sum_k A[m][k] B[n][k].
//
// Two ways to multiply:
//   codes: the 8-bit matrix instruction over 128 entries, which takes the scales as operands, a byte (exponent + 127) for every row of
//     either operand: a block of 128 is one instruction and its scaling costs nothing.  Inside, it adds products in groups of eight
//     and there loses what lies below 2^-13 of the group's largest (measured: 1 + 2^-13 is kept, 1 + 2^-14 is 1; over random operands
//     the result is 0.8e-5 to 1.5e-5 off in the 2-norm), the sums of groups are fp32.
//   values: codes become bf16 values with their scale already on, two in an instruction (a code has at most four significant bits, so
//     this is exact from bf16's last place, 2^-133, to its largest number), and the bf16 matrix instruction adds them in fp32 (2e-8
//     off).  Half the rate of the other: every fp8 instruction of this chip, with scales or without, adds in the same groups.
// Results in fp32 are products of values.  Results in bf16, which are off by up to 2^-8 anyway, are products of codes in the tiles, where
// the matrix instructions' rate counts (2048 x 4096 x 4096 in 36 us, of values 58), and of values with few rows, where it does not (one
// row by 4096 x 4096 4.8 us of codes and 4.9 of values, 32 rows 8.3 and 8.4, 64 rows 10.4 and 10.7), but of rows with scales beyond bf16's
// range.
// Both operands are read with one assignment of a lane's registers to positions inside a block; which it is does not matter to a
// sum over the block.  Rows are whole blocks (filled up with zeros), so the reduction has no tail; rows behind the last are read
// as the last one and not stored: a row of the result depends on its own row of A and its own row of B alone.
#pragma once
#include <type_traits>

#include "fp8_codes.h"
#include "fp8_plan.h"
#include "gemm_core.h"

struct Fp8Product {
    const uint8_t *a, *sa, *b, *sb;
    int M, N, nk;        // nk: blocks of the reduction
    int64_t ld, lds;     // bytes of a row of codes, of scales
    void *out;
};

// fp8_gemm_bf16.hip, fp8_gemm_f32.hip: the product with results of that type; ws: fp32 [slices][M][N] where there are several
int q8t_fp8_product_bf16(const Fp8Product &p, int fa, int fb, const Fp8Plan &plan, void *ws, hipStream_t st);
int q8t_fp8_product_f32(const Fp8Product &p, int fa, int fb, const Fp8Plan &plan, void *ws, hipStream_t st);

namespace {

typedef Fp8Product Product;

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
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

// Whether one of four stored scales may bring codes out of bf16's range: below its last place, 2^-133, or to 2^128 (e5m2's least code is
// 2^-16, its largest 1.75 * 2^15; e4m3's lie between).
__device__ __forceinline__ bool beyond_bf16(uint32_t scales)
{
    bool far = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) far |= (scales >> (8 * i) & 255u) - 10u > 229u;
    return far;
}

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

// four results of one row next to each other
template <class OUT>
__device__ __forceinline__ void store4(OUT *out, int64_t at, const f32x4 v, int count)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < count) out[at + i] = (OUT)v[i];
}

// Operands straight from memory to registers; the wavefronts of a workgroup share a tile of 16*MT x 16*NT results and take turns at
// the reduction, four blocks at a time, because four scales of a row are one word.  Products of values, for bf16 results
// but of rows with scales beyond bf16's range.  Bound by the weights' bytes: one row by 4096 x 4096 in 4.6 us, by 8192 x 8192 in 12.3
// (5.5 TB/s).
constexpr int kDirectWaves = 8;
template <int FA, int FB, class OUT, int MT, int NT>
__global__ __launch_bounds__(64 * kDirectWaves, (MT * NT == 1 ? 8 : 4)) void direct(const Product p)
{
    constexpr int W = kDirectWaves;
    __shared__ f32x4 fold[W][MT * NT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, r = lane & 15, g = lane / 16;
    const int n0 = blockIdx.x * (16 * NT), m0 = blockIdx.y * (16 * MT);
    bool fa[MT] = {}, fb[NT] = {};
    auto reduce = [&](auto wide, f32x4 (&acc)[MT][NT]) {
        constexpr bool WIDE = decltype(wide)::value;
        int row0 = r;
        asm volatile("" : "+v"(row0));   // addresses of its own: kept from one call for another they would take registers from the first
        const uint8_t *pa[MT], *psa[MT], *pb[NT], *psb[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int64_t row = min(m0 + 16 * i + row0, p.M - 1);
            pa[i] = p.a + row * p.ld + g * 16;
            psa[i] = p.sa + row * p.lds;
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int64_t row = min(n0 + 16 * j + row0, p.N - 1);
            pb[j] = p.b + row * p.ld + g * 16;
            psb[j] = p.sb + row * p.lds;
        }
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
            if (!WIDE || std::is_same<OUT, float>::value) continue;
#pragma unroll
            for (int i = 0; i < MT; ++i) fa[i] |= beyond_bf16(sa[i]);
#pragma unroll
            for (int j = 0; j < NT; ++j) fb[j] |= beyond_bf16(sb[j]);
        }
    };
    f32x4 acc[MT][NT];
    reduce(std::true_type(), acc);
    if (!std::is_same<OUT, float>::value) {   // rows with such scales once more, as codes; the others' results are their own
        bool any = false;
#pragma unroll
        for (int i = 0; i < MT; ++i) any |= fa[i];
#pragma unroll
        for (int j = 0; j < NT; ++j) any |= fb[j];
        if (__any(any)) {
            f32x4 far[MT][NT];
            reduce(std::false_type(), far);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const uint32_t rows = (uint32_t)__ballot(fb[j]) >> (4 * g);   // bit e: of row 4 * g + e
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = fa[i] || (rows >> e & 1u) ? far[i][j][e] : acc[i][j][e];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) fold[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            if ((i * NT + j) % W != wave) continue;   // the tiles are dealt out to the wavefronts
            f32x4 v = fold[0][i * NT + j][lane];
#pragma unroll
            for (int w = 1; w < W; ++w) v += fold[w][i * NT + j][lane];
            const int m = m0 + 16 * i + r, n = n0 + 16 * j + 4 * g;
            if (m < p.M) store4((OUT *)p.out, (int64_t)m * p.N + n, v, p.N - n);
        }
}

// ---- tiles staged in LDS ----------------------------------------------------------------------------------------
// BM x BN results a workgroup, WM x WN a wavefront in tiles of 32 x 32.  A step is one block of 128 of the reduction: BM + BN rows of
// 128 bytes that are copied to LDS past the registers, into one of two slots.  The last part of a step is multiplied out of
// registers while the first part of the next step is read and the slot just read is filled with the step behind that.  Piece s of LDS
// row r holds the 16 bytes s ^ perm(r) of the row's block, which keeps the fragment reads free of bank conflicts.  The scales of four
// steps are a word a row and go to LDS beside them.
// 8192 cubed: bf16 in 465 us (2.4 PFLOP/s), fp32 in 760 to 820 (1.34 to 1.45), tiles of 256 x 256, bound by the matrix instructions at the
// clock that the power leaves (1.77 GHz; busy 75 % of the cycles to fp32).  2048 x 4096 x 4096 to bf16 in 35 to 36 us among other calls and
// 38 to 46 on an idle card, tiles of 128 x 128, bound by the copies.
template <int BM_, int BN_, int WM_, int WN_, int SLOTS_>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, SLOTS = SLOTS_, MT = WM / 32, NT = WN / 32;
    static constexpr int WR = BM / WM, WC = BN / WN, WAVES = WR * WC, THREADS = 64 * WAVES;
    static constexpr int CA = BM / 8 / WAVES, CB = BN / 8 / WAVES;   // copies of eight rows that a wavefront makes a step
    static constexpr int SG = (BM + BN) / 64, CS = (SG + WAVES - 1) / WAVES;   // copies of 64 rows' scales
    static constexpr int COPIES = CA + CB + CS;
    static constexpr int SLOT = (BM + BN) * 128, SCALES = (BM + BN) * 4;
    static constexpr int LDS = SLOTS * SLOT + 2 * SCALES;
    static_assert(SLOTS == 2 || SLOTS == 4, "the scales of a step that is copied lie in this group of four steps or the next");
    static constexpr int BEHIND = (SLOTS - 2) * COPIES;   // copies that may be under way when a step's have to be there
    static constexpr int PER_SIMD = LDS > 80 * 1024 ? (WAVES + 3) / 4 : 2 * ((WAVES + 3) / 4);   // wavefronts
};

// 16 (4) bytes a lane from base + offset to lds + 16 (4) * lane, base and lds uniform in the wavefront; counted by its vmcnt
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy16(const uint8_t *base, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void copy4(const uint8_t *base, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop

// The part of a step that is multiplied at a time, as it comes out of LDS: half a block for the 8-bit instruction, a quarter where the
// codes become bf16 first.
template <bool WIDE>
struct Piece;
template <>
struct Piece<false> {
    static constexpr int SUBS = 2, READS = 2;
    i32x4 v[2];
    __device__ __forceinline__ void read(const uint8_t *row, int swizzle, int sub, int k)   // swizzle: perm ^ 2 * (lane / 32)
    {
        v[k] = *reinterpret_cast<const i32x4 *>(row + ((swizzle ^ (4 * sub + k)) * 16));
    }
    __device__ __forceinline__ i32x8 all() const { return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7); }
};
template <>
struct Piece<true> {
    static constexpr int SUBS = 4, READS = 1;
    i32x4 v[1];
    __device__ __forceinline__ void read(const uint8_t *row, int swizzle, int sub, int)   // swizzle: perm ^ (lane / 32)
    {
        v[0] = *reinterpret_cast<const i32x4 *>(row + ((swizzle ^ (2 * sub)) * 16));
    }
};
template <int FMT>
struct Widened {
    bf16x8 v[2];
    __device__ __forceinline__ void set(const Piece<true> &p, int scale)
    {
        const float s = __uint_as_float((uint32_t)scale << 23);
        v[0] = widen<FMT>(p.v[0][0], p.v[0][1], s);
        v[1] = widen<FMT>(p.v[0][2], p.v[0][3], s);
    }
};

// The products of one part, a tile of 32 x 32 at a time; between(t) is what the wavefront issues behind tile t while that is
// multiplied (loads of what comes next), pinned there: left to itself the compiler gathers all products in one place.
template <int FP, int FQ, class C, class F>
__device__ __forceinline__ void multiply(const Piece<false> (&p)[C::NT], const Piece<false> (&q)[C::MT], const int (&sp)[C::NT],
                                         const int (&sq)[C::MT], f32x16 (&acc)[C::MT][C::NT], F between)
{
#pragma unroll
    for (int i = 0; i < C::MT; ++i)
#pragma unroll
        for (int j = 0; j < C::NT; ++j) {
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(p[j].all(), q[i].all(), acc[i][j], FP, FQ, 0, sp[j], 0, sq[i]);
            between(i * C::NT + j);
            __builtin_amdgcn_sched_barrier(0);
        }
}
template <int FP, int FQ, class C, class F>
__device__ __forceinline__ void multiply(const Piece<true> (&p)[C::NT], const Piece<true> (&q)[C::MT], const int (&sp)[C::NT],
                                         const int (&sq)[C::MT], f32x16 (&acc)[C::MT][C::NT], F between)
{
    Widened<FP> b[C::NT];
    Widened<FQ> a[2];
    b[0].set(p[0], sp[0]);
    a[0].set(q[0], sq[0]);
#pragma unroll
    for (int i = 0; i < C::MT; ++i)
#pragma unroll
        for (int j = 0; j < C::NT; ++j) {
#pragma unroll
            for (int h = 0; h < 2; ++h) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[j].v[h], a[i & 1].v[h], acc[i][j], 0, 0, 0);
            // what the next tile needs is widened while this one is multiplied
            if (i == 0 && j + 1 < C::NT) b[j + 1].set(p[j + 1], sp[j + 1]);
            if (j + 1 == C::NT && i + 1 < C::MT) a[(i + 1) & 1].set(q[i + 1], sq[i + 1]);
            between(i * C::NT + j);
            __builtin_amdgcn_sched_barrier(0);
        }
}

// OUT: what is stored: the result, or fp32 partial sums of a slice of the reduction
template <int FA, int FB, bool WIDE, class OUT, class C>
__global__ __launch_bounds__(C::THREADS, C::PER_SIMD) void tiles(const Product p, int tm, int tn, int steps_per)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int total = tm * tn, logical = q8t_gemm::xcd_logical(blockIdx.x, total);
    if (logical >= total) return;
    // tiles in blocks of eight rows of tiles: those that an XCD works on at a time share both operands
    const int per = 8 * tn, blk = logical / per, in = logical - blk * per, bh = min(8, tm - blk * 8);
    const int m0 = (blk * 8 + in % bh) * C::BM, n0 = (in / bh) * C::BN;
    const int wr = wave % C::WR, wc = wave / C::WR;
    const int first = blockIdx.y * steps_per, steps = min(steps_per, p.nk - first);

    const uint8_t *ga = p.a + (int64_t)m0 * p.ld + (int64_t)first * 128, *gb = p.b + (int64_t)n0 * p.ld + (int64_t)first * 128;
    const uint8_t *gsa = p.sa + (int64_t)m0 * p.lds + first, *gsb = p.sb + (int64_t)n0 * p.lds + first;
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem;
    uint32_t oa[C::CA], ob[C::CB], os[C::CS];
#pragma unroll
    for (int c = 0; c < C::CA; ++c) {
        const int r = (c * C::WAVES + wave) * 8 + lane / 8;
        oa[c] = (uint32_t)((min(m0 + r, p.M - 1) - m0) * p.ld) + (((lane & 7) ^ ((r >> 1) & 7)) * 16);
    }
#pragma unroll
    for (int c = 0; c < C::CB; ++c) {
        const int r = (c * C::WAVES + wave) * 8 + lane / 8;
        ob[c] = (uint32_t)((min(n0 + r, p.N - 1) - n0) * p.ld) + (((lane & 7) ^ ((r >> 1) & 7)) * 16);
    }
#pragma unroll
    for (int c = 0; c < C::CS; ++c) {
        const int g = min(c * C::WAVES + wave, C::SG - 1), r = g * 64 + lane;
        const int row = g >= C::BM / 64 ? min(n0 + r - C::BM, p.N - 1) - n0 : min(m0 + r, p.M - 1) - m0;
        os[c] = (uint32_t)(row * p.lds);
    }
    // Copy c of step s.  Steps behind the last are asked for too and read the last one again, into slots that nobody reads, so that
    // the loop has no branches.  The word with a step's scales is copied with each of its four steps, over itself.
    auto copy = [&](int s, int c) {
        const uint32_t to = base + (s & (C::SLOTS - 1)) * C::SLOT;
        s = min(s, steps - 1);
        if (c < C::CA) {
            copy16(ga + (int64_t)s * 128, oa[c], to + (c * C::WAVES + wave) * 1024);
        } else if (c < C::CA + C::CB) {
            copy16(gb + (int64_t)s * 128, ob[c - C::CA], to + C::BM * 128 + ((c - C::CA) * C::WAVES + wave) * 1024);
        } else {
            const int d = c - C::CA - C::CB, g = min(d * C::WAVES + wave, C::SG - 1);
            copy4((g >= C::BM / 64 ? gsb : gsa) + (s & ~3), os[d], base + C::SLOTS * C::SLOT + ((s >> 2) & 1) * C::SCALES + g * 256);
        }
    };

    const int r32 = lane & 31, half = lane / 32, perm = (r32 >> 1) & 7, swizzle = perm ^ (WIDE ? half : 2 * half);
    const uint8_t *rowa = smem + (wr * C::WM + r32) * 128, *rowb = smem + (C::BM + wc * C::WN + r32) * 128;
    const uint8_t *sca = smem + C::SLOTS * C::SLOT + (wr * C::WM + r32) * 4, *scb = smem + C::SLOTS * C::SLOT + (C::BM + wc * C::WN + r32) * 4;
    constexpr int SUBS = Piece<WIDE>::SUBS, PR = Piece<WIDE>::READS, READS = (C::MT + C::NT) * PR, TILES = C::MT * C::NT;
    Piece<WIDE> fa[2][C::MT], fb[2][C::NT];
    int sa[C::MT], sb[C::NT], na[C::MT], nb[C::NT];
    auto read = [&](int s, int sub, int c) {   // read c of a part, in the order in which the products need them
        const int at = (s & (C::SLOTS - 1)) * C::SLOT, f = c / PR, into = sub & 1;
        if (f == 0 || f > C::NT) {
            const int i = f == 0 ? 0 : f - C::NT;
            fa[into][i].read(rowa + at + i * 32 * 128, swizzle, sub, c % PR);
        } else {
            fb[into][f - 1].read(rowb + at + (f - 1) * 32 * 128, swizzle, sub, c % PR);
        }
    };
    auto scale = [&](int s, int c) {   // of block s
        const int at = ((s >> 2) & 1) * C::SCALES + (s & 3);
        if (c < C::MT) na[c] = sca[at + c * 128];
        else nb[c - C::MT] = scb[at + (c - C::MT) * 128];
    };
    f32x16 acc[C::MT][C::NT];
#pragma unroll
    for (int i = 0; i < C::MT; ++i)
#pragma unroll
        for (int j = 0; j < C::NT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

    // all that the next copies overwrite has been read, and the next step's copies are there
    auto meet = [] { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(C::BEHIND) : "memory"); };
#pragma unroll
    for (int k = 0; k < C::SLOTS - 1; ++k)
#pragma unroll
        for (int c = 0; c < C::COPIES; ++c) copy(k, c);
    meet();
#pragma unroll
    for (int c = 0; c < C::COPIES; ++c) copy(C::SLOTS - 1, c);
#pragma unroll
    for (int c = 0; c < C::MT + C::NT; ++c) scale(0, c);
#pragma unroll
    for (int c = 0; c < READS; ++c) read(0, 0, c);
    auto step = [&](int s, auto last) {
        constexpr bool LAST = decltype(last)::value;
#pragma unroll
        for (int i = 0; i < C::MT; ++i) sa[i] = na[i];
#pragma unroll
        for (int j = 0; j < C::NT; ++j) sb[j] = nb[j];
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
            if (sub == SUBS - 1 && !LAST) meet();
            __builtin_amdgcn_sched_barrier(0);
            multiply<FB, FA, C>(fb[sub & 1], fa[sub & 1], sb, sa, acc, [&](int t) {
                if (sub < SUBS - 1) {
#pragma unroll
                    for (int c = t * READS / TILES; c < (t + 1) * READS / TILES; ++c) read(s, sub + 1, c);
                } else if (!LAST) {
                    // copies first: they have until the next meeting
                    constexpr int PER = (C::COPIES + TILES - 1) / TILES;
#pragma unroll
                    for (int c = t * PER; c < (t + 1) * PER && c < C::COPIES; ++c) copy(s + C::SLOTS, c);
#pragma unroll
                    for (int c = t * READS / TILES; c < (t + 1) * READS / TILES; ++c) read(s + 1, 0, c);
#pragma unroll
                    for (int c = t * (C::MT + C::NT) / TILES; c < (t + 1) * (C::MT + C::NT) / TILES; ++c) scale(s + 1, c);
                }
            });
        }
    };
    for (int s = 0; s < steps - 1; ++s) step(s, std::false_type());
    step(steps - 1, std::true_type());

    // Results go through LDS, 32 rows of the wavefront at a time, so that rows leave in pieces of 16 bytes a lane.
    constexpr int ROW = C::WN * sizeof(OUT) + 16, PP = C::WN * sizeof(OUT) / 16, PER = 16 / sizeof(OUT);
    static_assert(C::WAVES * 32 * ROW <= C::LDS, "the staged results fit");
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    uint8_t *stage = smem + wave * 32 * ROW;
    OUT *out = (OUT *)p.out + (int64_t)blockIdx.y * p.M * p.N;
#pragma unroll
    for (int i = 0; i < C::MT; ++i) {
        const int mi = m0 + wr * C::WM + i * 32;
#pragma unroll
        for (int j = 0; j < C::NT; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {   // four results next to each other
                uint8_t *to = stage + r32 * ROW + (j * 32 + g * 8 + half * 4) * sizeof(OUT);
                const f32x16 &v = acc[i][j];
                if (sizeof(OUT) == 4) *reinterpret_cast<f32x4 *>(to) = f32x4{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
                else *reinterpret_cast<uint2 *>(to) = make_uint2(q8t_pack_bf16(v[4 * g], v[4 * g + 1]), q8t_pack_bf16(v[4 * g + 2], v[4 * g + 3]));
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int k = 0; k < 32 * PP / 64; ++k) {
            const int t = k * 64 + lane, r = t / PP, c = t % PP, m = mi + r, n = n0 + wc * C::WN + c * PER;
            typedef typename Q8tRaw<sizeof(OUT)>::type raw;
            const uint4 v = *reinterpret_cast<const uint4 *>(stage + r * ROW + c * 16);
            if (m < p.M && n < p.N) {
                OUT *to = out + (int64_t)m * p.N + n;
                if (n + PER <= p.N) {
                    *reinterpret_cast<raw *>(to) = raw{v.x, v.y, v.z, v.w};
                } else {
                    const OUT *e = reinterpret_cast<const OUT *>(stage + r * ROW + c * 16);
                    for (int x = 0; x < p.N - n; ++x) to[x] = e[x];
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
        __builtin_amdgcn_wave_barrier();
    }
}

template <int FA, int FB, bool WIDE, class OUT, class C>
int run_tiles(Product p, int slices, void *ws, hipStream_t st)
{
    static Q8tLdsOptIn opt;
    const int rc = q8t_allow_lds(opt, (const void *)tiles<FA, FB, WIDE, OUT, C>, C::LDS);
    if (rc) return rc;
    const int tm = (p.M + C::BM - 1) / C::BM, tn = (p.N + C::BN - 1) / C::BN;
    const int steps = ((p.nk + slices - 1) / slices + 3) & ~3;   // whole words of scales
    if (slices > 1) p.out = ws;
    tiles<FA, FB, WIDE, OUT, C><<<dim3(q8t_gemm::xcd_grid((int64_t)tm * tn), (p.nk + steps - 1) / steps), C::THREADS, C::LDS, st>>>(p, tm, tn, steps);
    Q8T_LAUNCH_CHECK();
    return Q8T_OK;
}

// sum over the slices, in their order
template <class OUT>
__global__ __launch_bounds__(256) void fold_slices(const float *__restrict__ part, int slices, int64_t n, OUT *__restrict__ out)
{
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (i >= n) return;
    const int count = n - i >= 8 ? 8 : (int)(n - i);
    float v[8], w[8];
    q8t_load8<float, false>(part + i, v, count);
    for (int z = 1; z < slices; ++z) {
        q8t_load8<float, false>(part + z * n + i, w, count);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += w[k];
    }
    q8t_store8(out + i, v, count);
}
template <class OUT>
int run_fold(const Product &p, int slices, const void *ws, hipStream_t st)
{
    const int steps = ((p.nk + slices - 1) / slices + 3) & ~3;
    const int64_t n = (int64_t)p.M * p.N;
    fold_slices<OUT><<<(unsigned)((n + 2047) / 2048), 256, 0, st>>>((const float *)ws, (p.nk + steps - 1) / steps, n, (OUT *)p.out);
    Q8T_LAUNCH_CHECK();
    return Q8T_OK;
}

template <int FA, int FB, class OUT, int MT, int NT>
int run_direct(const Product &p, hipStream_t st)
{
    direct<FA, FB, OUT, MT, NT><<<dim3((p.N + 16 * NT - 1) / (16 * NT), (p.M + 16 * MT - 1) / (16 * MT)), 64 * kDirectWaves, 0, st>>>(p);
    Q8T_LAUNCH_CHECK();
    return Q8T_OK;
}

template <class R>
int by_format(int fa, int fb, R run)
{
    typedef std::integral_constant<int, Q8T_E4M3> E4;
    typedef std::integral_constant<int, Q8T_E5M2> E5;
    if (fa == Q8T_E4M3) return fb == Q8T_E4M3 ? run(E4(), E4()) : run(E4(), E5());
    return fb == Q8T_E4M3 ? run(E5(), E4()) : run(E5(), E5());
}

}  // namespace
