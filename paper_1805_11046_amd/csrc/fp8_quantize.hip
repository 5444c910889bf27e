// fp8 quantization with a scale for each block of 128: q8t_fp8_quantize (formats, scales and roundings in fp8_codes.h).
#include "fp8_codes.h"

namespace {

constexpr int kThreads = 256;

// Row copy alone: a block of 128 belongs to 16 lanes of eight entries each.
template <class T, int FMT, bool STOCH, bool ALIGNED>
__global__ __launch_bounds__(kThreads) void quantize_rows(const T *__restrict__ x, uint32_t nblocks, uint32_t nb, int64_t C, uint64_t seed,
                                                          const int64_t *__restrict__ step, uint8_t *__restrict__ q,
                                                          uint8_t *__restrict__ s)
{
    const uint32_t g = blockIdx.x * (kThreads / 16) + threadIdx.x / 16, lane = threadIdx.x & 15;
    if (g >= nblocks) return;
    const uint32_t row = g / nb, kb = g - row * nb;
    const int64_t c = (int64_t)kb * 128 + lane * 8, at = (int64_t)row * C + c;
    const int64_t left = C - c;
    float v[8];
    uint32_t r[4];
    q8t_load8(x + at, v, left >= 8 ? 8 : (int)left);
    if (STOCH) q8t_draw8<ALIGNED>(at, q8t_seed(seed, step), r);
    const uint32_t scale = fp8_scale<FMT>(fp8_max16(fp8_max8(v)));
    const uint2 w = fp8_codes8<FMT, STOCH>(v, scale, r);
    *reinterpret_cast<uint2 *>(q + (int64_t)row * nb * 128 + c) = w;
    const uint32_t sp = (nb + 3) & ~3u;
    if (lane == 0) s[(int64_t)row * sp + kb] = (uint8_t)scale;
    if (kb == nb - 1 && lane > 0 && kb + lane < sp) s[(int64_t)row * sp + kb + lane] = 127;
}

// Both copies of a 128 x 128 tile from one read; every thread holds a patch of 8 x 8, so that it packs eight codes along
// either axis.  SQUARE: one scale for the tile, and the transposed copy holds the same codes.
template <class T, int FMT, bool STOCH, bool ALIGNED, bool SQUARE>
__global__ __launch_bounds__(kThreads) void quantize_tile(const T *__restrict__ x, int64_t R, int64_t C, uint32_t nbr, uint32_t nbc,
                                                          uint64_t seed, const int64_t *__restrict__ step, uint8_t *__restrict__ q,
                                                          uint8_t *__restrict__ s, uint8_t *__restrict__ qt, uint8_t *__restrict__ st)
{
    __shared__ uint32_t colmax[4][128];
    __shared__ __align__(16) uint8_t turned[128][144];
    const uint32_t tr = blockIdx.x / nbc, tc = blockIdx.x - tr * nbc;
    const int ty = threadIdx.x / 16, tx = threadIdx.x & 15, wave = threadIdx.x / 64;
    const int64_t r0 = (int64_t)tr * 128 + ty * 8, c0 = (int64_t)tc * 128 + tx * 8;
    const int cols = (int)min((int64_t)8, C - c0);
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (r0 + i < R) {
            q8t_load8(x + (r0 + i) * C + c0, v[i], cols);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
        }
    }
    uint32_t rmax[8], cmax[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) cmax[j] = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        rmax[i] = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t m = fp8_magnitude(v[i][j]);
            rmax[i] = max(rmax[i], m);
            cmax[j] = max(cmax[j], m);
        }
    }
    if (SQUARE) {
        uint32_t m = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, rmax[i]);
        m = fp8_max16(m);
        m = max(m, (uint32_t)__shfl_xor((int)m, 16, 64));
        m = max(m, (uint32_t)__shfl_xor((int)m, 32, 64));
        if ((threadIdx.x & 63) == 0) colmax[wave][0] = m;
        __syncthreads();
        m = max(max(colmax[0][0], colmax[1][0]), max(colmax[2][0], colmax[3][0]));
#pragma unroll
        for (int i = 0; i < 8; ++i) rmax[i] = cmax[i] = m;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) rmax[i] = fp8_max16(rmax[i]);
        if (qt) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                cmax[j] = max(cmax[j], (uint32_t)__shfl_xor((int)cmax[j], 16, 64));
                cmax[j] = max(cmax[j], (uint32_t)__shfl_xor((int)cmax[j], 32, 64));
                if ((ty & 3) == 0) colmax[wave][tx * 8 + j] = cmax[j];
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = tx * 8 + j;
                cmax[j] = max(max(colmax[0][c], colmax[1][c]), max(colmax[2][c], colmax[3][c]));
            }
        }
    }
    const uint32_t sp = (nbc + 3) & ~3u, spt = (nbr + 3) & ~3u;
    const Q8tSeed sd = STOCH ? q8t_seed(seed, step) : Q8tSeed{0, 0};
    // one byte of a code a column and row: patch[j] gathers column j's eight codes
    uint2 patch[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) patch[j] = make_uint2(0u, 0u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint32_t r[4];
        if (STOCH) q8t_draw8<ALIGNED>((r0 + i) * C + c0, sd, r);
        const uint32_t scale = fp8_scale<FMT>(rmax[i]);
        const uint2 w = fp8_codes8<FMT, STOCH>(v[i], scale, r);
        if (r0 + i < R) {
            *reinterpret_cast<uint2 *>(q + (r0 + i) * nbc * 128 + c0) = w;
            if (tx == 0) s[(r0 + i) * sp + tc] = (uint8_t)scale;
            if (tc == nbc - 1 && tx > 0 && tc + tx < sp) s[(r0 + i) * sp + tc + tx] = 127;
        }
        if (!qt) continue;
        uint2 t = w;
        if (!SQUARE) {   // the column's scales
            uint32_t code[8];
            if (STOCH) {
#pragma unroll
                for (int j = 0; j < 8; ++j) code[j] = fp8_stochastic<FMT>(v[i][j] * fp8_inverse(fp8_scale<FMT>(cmax[j])), q8t_draw(r, j));
                t.x = code[0] | code[1] << 8 | code[2] << 16 | code[3] << 24;
                t.y = code[4] | code[5] << 8 | code[6] << 16 | code[7] << 24;
            } else {
                float u[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] = v[i][j] * fp8_inverse(fp8_scale<FMT>(cmax[j]));
                t.x = fp8_pack2<FMT, true>(u[2], u[3], fp8_pack2<FMT, false>(u[0], u[1], 0u));
                t.y = fp8_pack2<FMT, true>(u[6], u[7], fp8_pack2<FMT, false>(u[4], u[5], 0u));
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t b = ((j < 4 ? t.x : t.y) >> (8 * (j & 3))) & 255u;
            if (i < 4) patch[j].x |= b << (8 * i);
            else patch[j].y |= b << (8 * (i - 4));
        }
    }
    if (!qt) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) *reinterpret_cast<uint2 *>(&turned[tx * 8 + j][ty * 8]) = patch[j];
    if (ty == 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c0 + j < C) st[(c0 + j) * spt + tr] = (uint8_t)fp8_scale<FMT>(cmax[j]);
    }
    if (tr == nbr - 1 && tr + ty < spt && ty > 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c0 + j < C) st[(c0 + j) * spt + tr + ty] = 127;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int piece = k * kThreads + threadIdx.x, col = piece / 8, at = (piece & 7) * 16;
        const int64_t c = (int64_t)tc * 128 + col;
        if (c < C) *reinterpret_cast<uint4 *>(qt + c * nbr * 128 + (int64_t)tr * 128 + at) = *reinterpret_cast<const uint4 *>(&turned[col][at]);
    }
}

struct Args {
    const void *x;
    int64_t R, C;
    uint64_t seed;
    const int64_t *step;
    uint8_t *q, *s, *qt, *st;
    hipStream_t stream;
};

template <class T, int FMT, bool STOCH, bool ALIGNED>
int launch(const Args &a, bool square)
{
    const uint32_t nbr = (uint32_t)((a.R + 127) / 128), nbc = (uint32_t)((a.C + 127) / 128);
    if (!square && !a.qt) {
        const uint32_t blocks = (uint32_t)(a.R * nbc);
        quantize_rows<T, FMT, STOCH, ALIGNED><<<(blocks + 15) / 16, kThreads, 0, a.stream>>>((const T *)a.x, blocks, nbc, a.C, a.seed,
                                                                                           a.step, a.q, a.s);
    } else if (square) {
        quantize_tile<T, FMT, STOCH, ALIGNED, true><<<nbr * nbc, kThreads, 0, a.stream>>>((const T *)a.x, a.R, a.C, nbr, nbc, a.seed,
                                                                                       a.step, a.q, a.s, a.qt, a.st);
    } else {
        quantize_tile<T, FMT, STOCH, ALIGNED, false><<<nbr * nbc, kThreads, 0, a.stream>>>((const T *)a.x, a.R, a.C, nbr, nbc, a.seed,
                                                                                        a.step, a.q, a.s, a.qt, a.st);
    }
    Q8T_LAUNCH_CHECK();
    return Q8T_OK;
}
template <class T, int FMT>
int choose(const Args &a, bool square, bool stochastic)
{
    if (!stochastic) return launch<T, FMT, false, true>(a, square);
    return a.C % 4 == 0 ? launch<T, FMT, true, true>(a, square) : launch<T, FMT, true, false>(a, square);
}

}  // namespace

extern "C" int q8t_fp8_quantize(const void *x, int type, int64_t rows, int64_t cols, int format, int square, int stochastic, uint64_t seed,
                                const int64_t *step, uint8_t *q, uint8_t *s, uint8_t *qt, uint8_t *st, void *stream)
{
    if (rows < 0 || cols < 0) return Q8T_ERR_SHAPE;
    if ((type != Q8T_F32 && type != Q8T_BF16) || (format != Q8T_E4M3 && format != Q8T_E5M2)) return Q8T_ERR_VALUE;
    if (rows == 0 || cols == 0) return Q8T_OK;
    // a launch holds fewer than 2^32 threads, 16 for a block of either copy; the generator counts groups of four in 32 bits
    const int64_t most = (int64_t)1 << 28, wide = (int64_t)1 << 31;
    if (rows >= wide || cols >= wide || rows > ((int64_t)1 << 34) / cols) return Q8T_ERR_SHAPE;
    if (rows * ((cols + 127) / 128) >= most || cols * ((rows + 127) / 128) >= most) return Q8T_ERR_SHAPE;
    if (!x || !q || !s || !qt != !st) return Q8T_ERR_NULL;
    if (!q8t_aligned(q, 16) || (qt && !q8t_aligned(qt, 16))) return Q8T_ERR_SHAPE;
    const Args a = {x, rows, cols, seed, step, q, s, qt, st, (hipStream_t)stream};
    if (type == Q8T_F32)
        return format == Q8T_E4M3 ? choose<float, Q8T_E4M3>(a, square, stochastic) : choose<float, Q8T_E5M2>(a, square, stochastic);
    return format == Q8T_E4M3 ? choose<q8t_bf16, Q8T_E4M3>(a, square, stochastic) : choose<q8t_bf16, Q8T_E5M2>(a, square, stochastic);
}
