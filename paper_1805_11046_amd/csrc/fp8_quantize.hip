// fp8 quantization with a scale for each block of 128: q8t_fp8_quantize (formats, scales and roundings in fp8_codes.h).
#include "fp8_codes.h"

namespace {

constexpr int kThreads = 256;

// Row copy alone: a block of 128 belongs to 16 lanes of eight entries each.  Bound by memory: 4096 x 4096 from fp32 in 16.1 us, from bf16
// in 11.5, which is 15 % over a copy's time for as many bytes; stochastic by the generator's products, 17.2.
template <class T, int FMT, bool STOCH, bool ALIGNED>
__global__ __launch_bounds__(kThreads) void quantize_rows(const T *__restrict__ x, uint32_t nblocks, uint32_t nb, int64_t C, uint64_t seed,
                                                          const int64_t *__restrict__ step, uint8_t *__restrict__ q,
                                                          uint8_t *__restrict__ s)
{
    const uint32_t g = blockIdx.x * (kThreads / 16) + threadIdx.x / 16, lane = threadIdx.x & 15;
    if (g >= nblocks) return;
    const uint32_t row = g / nb, kb = g - row * nb;
    const int64_t c = (int64_t)kb * 128 + lane * 8, at = (int64_t)row * C + c;
    Q8tEight<T> e;
    if (C < 8) {
        e.few(x + (int64_t)row * C, lane == 0 ? (int)C : 0);
    } else {   // a row's last entries behind a multiple of eight: read from eight before its end
        e.template vector<true>(x + (int64_t)row * C + min(c, C - 8));
        if (c + 8 > C) e.template settle<false>((uint32_t)min(c + 8 - C, (int64_t)8), 8u);
    }
    float v[8];
    uint32_t r[4];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = e[j];
    if (STOCH) q8t_draw8<ALIGNED>(at, q8t_seed(seed, step), r);
    uint32_t scale[1] = {fp8_scale<FMT>(fp8_max16(fp8_max8(v)))};
    if (STOCH) fp8_round_up(scale);
    const uint2 w = fp8_codes8<FMT, STOCH>(v, scale[0], r);
    *reinterpret_cast<uint2 *>(q + (int64_t)row * nb * 128 + c) = w;
    const uint32_t sp = (nb + 3) & ~3u;
    if (lane == 0) s[(int64_t)row * sp + kb] = (uint8_t)scale[0];
    if (kb == nb - 1 && lane > 0 && kb + lane < sp) s[(int64_t)row * sp + kb + lane] = 127;
}

// Magnitudes of eight values and their maxima.  bf16: two in a word, as the upper halves of the fp32 patterns; whole numbers are
// ordered like the magnitudes either way.  An infinity or a NaN, which a block's scale does not count, is at least LIMIT.
template <class T>
struct Magnitudes;
template <>
struct Magnitudes<float> {
    static constexpr int N = 8;
    static constexpr uint32_t LIMIT = 0x7F800000u;
    static __device__ __forceinline__ uint32_t of(uint32_t w) { return w & 0x7FFFFFFFu; }
    static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b) { return max(a, b); }
    static __device__ __forceinline__ uint32_t finite(uint32_t m) { return m < LIMIT ? m : 0u; }
    static __device__ __forceinline__ uint32_t one(uint32_t m) { return m; }                       // the larger of the word's, as fp32
    static __device__ __forceinline__ uint32_t column(const uint32_t m[N], int j) { return m[j]; }   // column j's, as fp32
};
template <>
struct Magnitudes<q8t_bf16> {
    static constexpr int N = 4;
    static constexpr uint32_t LIMIT = 0x7F800000u;
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ uint32_t of(uint32_t w) { return w & 0x7FFF7FFFu; }
    static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b)
    {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
    }
    static __device__ __forceinline__ uint32_t finite(uint32_t m)
    {
        return ((m & 0xFFFFu) < 0x7F80u ? m & 0xFFFFu : 0u) | ((m >> 16) < 0x7F80u ? m & 0xFFFF0000u : 0u);
    }
    static __device__ __forceinline__ uint32_t one(uint32_t m) { return max(m & 0xFFFF0000u, m << 16); }
    static __device__ __forceinline__ uint32_t column(const uint32_t m[N], int j) { return (j & 1) ? m[j >> 1] & 0xFFFF0000u : m[j >> 1] << 16; }
};

// four signs as the codes have them
__device__ __forceinline__ uint32_t signs4(const Q8tEight<float> &x, int h)
{
    const uint32_t lo = __builtin_amdgcn_perm(x.w[4 * h + 1], x.w[4 * h], 0x00000703u), hi = __builtin_amdgcn_perm(x.w[4 * h + 3], x.w[4 * h + 2], 0x07030000u);
    return ((lo & 0xFFFFu) | (hi & 0xFFFF0000u)) & 0x80808080u;
}
__device__ __forceinline__ uint32_t signs4(const Q8tEight<q8t_bf16> &x, int h)
{
    return __builtin_amdgcn_perm(x.w[2 * h + 1], x.w[2 * h], 0x07050301u) & 0x80808080u;
}

// bytes of four words turned: o[i] byte k = w[k] byte i
__device__ __forceinline__ void turn4(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t o[4])
{
    const uint32_t p = __builtin_amdgcn_perm(b, a, 0x05010400u), q = __builtin_amdgcn_perm(b, a, 0x07030602u);
    const uint32_t r = __builtin_amdgcn_perm(d, c, 0x05010400u), s = __builtin_amdgcn_perm(d, c, 0x07030602u);
    o[0] = __builtin_amdgcn_perm(r, p, 0x05040100u);
    o[1] = __builtin_amdgcn_perm(r, p, 0x07060302u);
    o[2] = __builtin_amdgcn_perm(s, q, 0x05040100u);
    o[3] = __builtin_amdgcn_perm(s, q, 0x07060302u);
}

// Eight stochastic codes of one row under the scales of its eight columns (or the one of its block: the same for all j).
template <int FMT, class Draw>   // finite values, scales above -EMIN
__device__ __forceinline__ uint2 drawn8(const uint32_t m[8], const uint32_t drawn[8], const uint32_t signs[2], Draw draw)
{
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        w[h] = signs[h];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[h] |= draw(4 * h + i).code(m[4 * h + i], drawn[4 * h + i]) << (8 * i);
    }
    return make_uint2(w[0], w[1]);
}
template <int FMT, class T, class Scale>   // any
__device__ __forceinline__ uint2 any8(const Q8tEight<T> &x, const uint32_t drawn[8], Scale scale)
{
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j >> 2] |= fp8_drawn<FMT>(x[j], fp8_inverse(scale(j)), drawn[j]) << (8 * (j & 3));
    return make_uint2(w[0], w[1]);
}

// Both copies of a 128 x 128 tile from one read; every thread holds a patch of 8 x 8, so that it packs eight codes along
// either axis.  SQUARE: one scale for the tile, and the transposed copy holds the same codes.
// Bound by memory where the rounding is to nearest: both copies of 8192 x 8192 from bf16 in 51.5 us, the time of a copy of as many bytes;
// one scale a tile of 4096 x 4096 from fp32 in 24.3 for 20.  Stochastic 3001 x 5003 from bf16 in 25 us for 12: all tiles are on the card at
// once and read, compute and write together, so that memory (2.8 TB/s) and the vector unit (48 % of the cycles) wait for each other;
// 8192 x 8192, where rounds of tiles overlap, takes 68.1.  Half of the instructions are the generator's, in three groups of four for
// eight entries where a row starts inside a group (3008 x 5008 takes 2 us less).
template <class T, int FMT, bool STOCH, bool ALIGNED, bool SQUARE>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 2) void quantize_tile(const T *__restrict__ x, int64_t R, int64_t C, uint32_t nbr, uint32_t nbc,
                                                          uint64_t seed, const int64_t *__restrict__ step, uint8_t *__restrict__ q,
                                                          uint8_t *__restrict__ s, uint8_t *__restrict__ qt, uint8_t *__restrict__ st)
{
    typedef Magnitudes<T> Mag;
    constexpr int N = Mag::N;
    __shared__ uint32_t colmax[4][16][N];
    // the codes by columns, 16 bytes of rows in a piece; a patch's columns have their pieces in an order of their own, and columns from 64 on
    // lie half of the banks further, so that the lanes of a store have banks of their own; rows of 144 bytes: 27.1 us for 24.3 at 4096 x 4096 from fp32
    __shared__ __align__(16) uint8_t turned[129 * 128];
    auto place = [](int col, int piece) { return col * 128 + (col >> 6) * 128 + ((piece ^ (col >> 3 & 7)) << 4); };
    const uint32_t tr = blockIdx.x / nbc, tc = blockIdx.x - tr * nbc;
    const int ty = threadIdx.x / 16, tx = threadIdx.x & 15, wave = threadIdx.x / 64;
    const int64_t r0 = (int64_t)tr * 128 + ty * 8, c0 = (int64_t)tc * 128 + tx * 8;
    const int cols = (int)min((int64_t)8, C - c0), rows = (int)max((int64_t)0, min((int64_t)8, R - r0));
    // a row's last entries behind a multiple of eight: read from eight before its end, and put right once all rows are on their way
    const bool tiny = C < 8;
    Q8tEight<T> v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const T *row = x + (r0 + min(i, max(rows - 1, 0))) * C;   // rows behind the last are that one again, and cleared below
        if (rows <= 0) row = x;
        if (tiny) v[i].few(row, (int)C);
        else v[i].template vector<true>(row + min(c0, C - 8));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (cols < 8 && !tiny) v[i].template settle<false>((uint32_t)min(8 - cols, 8), 8u);   // as many to drop in front as are missing
        if ((tiny && tx > 0) || i >= rows) {
#pragma unroll
            for (int k = 0; k < N; ++k) v[i].w[k] = 0u;
        }
    }
    uint32_t rmax[8], cmax[N];
    auto maxima = [&](auto keep) {
#pragma unroll
        for (int k = 0; k < N; ++k) cmax[k] = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            rmax[i] = 0u;
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const uint32_t m = keep(Mag::of(v[i].w[k]));
                rmax[i] = Mag::most(rmax[i], m);
                cmax[k] = Mag::most(cmax[k], m);
            }
        }
    };
    maxima([](uint32_t m) { return m; });
    uint32_t all = 0u;
#pragma unroll
    for (int k = 0; k < N; ++k) all = Mag::most(all, cmax[k]);
    bool plain = Mag::one(all) < Mag::LIMIT;   // no infinity or NaN, and below: no scale at the lower end
    if (!plain) maxima([](uint32_t m) { return Mag::finite(m); });
    if (SQUARE) {
        uint32_t m = 0u;
#pragma unroll
        for (int k = 0; k < N; ++k) m = Mag::most(m, cmax[k]);
        m = fp8_max16(Mag::one(m));
        m = max(m, (uint32_t)__shfl_xor((int)m, 16, 64));
        m = max(m, (uint32_t)__shfl_xor((int)m, 32, 64));
        if ((threadIdx.x & 63) == 0) colmax[wave][0][0] = m;
        __syncthreads();
        rmax[0] = max(max(colmax[0][0][0], colmax[1][0][0]), max(colmax[2][0][0], colmax[3][0][0]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) rmax[i] = Mag::one(fp8_fold16(rmax[i], [](uint32_t a, uint32_t b) { return Mag::most(a, b); }));
        if (qt) {
#pragma unroll
            for (int k = 0; k < N; ++k) {
                cmax[k] = Mag::most(cmax[k], (uint32_t)__shfl_xor((int)cmax[k], 16, 64));
                cmax[k] = Mag::most(cmax[k], (uint32_t)__shfl_xor((int)cmax[k], 32, 64));
                if ((ty & 3) == 0) colmax[wave][tx][k] = cmax[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < N; ++k)
                cmax[k] = Mag::most(Mag::most(colmax[0][tx][k], colmax[1][tx][k]), Mag::most(colmax[2][tx][k], colmax[3][tx][k]));
        }
    }
    uint32_t cscale[8];   // stored scales of the columns
#pragma unroll
    for (int j = 0; j < 8; ++j) cscale[j] = fp8_scale<FMT>(SQUARE ? rmax[0] : Mag::column(cmax, j));
    uint32_t rscale[8];   // and of the rows
#pragma unroll
    for (int i = 0; i < 8; ++i) rscale[i] = fp8_scale<FMT>(rmax[SQUARE ? 0 : i]);
    if (STOCH) {
        uint32_t lowest = rscale[0];
#pragma unroll
        for (int i = 0; i < (SQUARE ? 0 : 8); ++i) lowest = min(lowest, min(rscale[i], cscale[i]));
        plain = plain && lowest > (uint32_t)-Fp8Format<FMT>::EMIN;
        fp8_round_up(rscale);
        fp8_round_up(cscale);
    }
    const uint32_t sp = (nbc + 3) & ~3u, spt = (nbr + 3) & ~3u;
    const Q8tSeed sd = STOCH ? q8t_seed(seed, step) : Q8tSeed{0, 0};
    uint2 across[8];   // rows of codes under the columns' scales
    auto store = [&](int i, uint2 w) { *reinterpret_cast<uint2 *>(q + (r0 + i) * nbc * 128 + c0) = w; };
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint2 w;
        if (STOCH) {
            uint32_t r[4], m[8], drawn[8];
            const uint32_t signs[2] = {signs4(v[i], 0), signs4(v[i], 1)};
            q8t_draw8<ALIGNED>((r0 + i) * C + c0, sd, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                m[j] = v[i].bits(j) & 0x7FFFFFFFu;
                drawn[j] = Fp8Draw<FMT>::drawn(q8t_draw(r, j));
            }
            if (plain) {
                const Fp8Draw<FMT> d(rscale[i]);
                w = drawn8<FMT>(m, drawn, signs, [&](int) { return d; });
                if (!SQUARE) across[i] = drawn8<FMT>(m, drawn, signs, [&](int j) { return Fp8Draw<FMT>(cscale[j]); });
            } else {
                w = any8<FMT>(v[i], drawn, [&](int) { return rscale[i]; });
                if (!SQUARE) across[i] = any8<FMT>(v[i], drawn, [&](int j) { return cscale[j]; });
            }
        } else {
            float f[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = v[i][j];
            w = fp8_codes8<FMT, false>(f, rscale[i], nullptr);
            if (!SQUARE && qt) {
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] *= fp8_inverse(cscale[j]);
                across[i].x = fp8_pack2<FMT, true>(f[2], f[3], fp8_pack2<FMT, false>(f[0], f[1], 0u));
                across[i].y = fp8_pack2<FMT, true>(f[6], f[7], fp8_pack2<FMT, false>(f[4], f[5], 0u));
            }
        }
        if (SQUARE) across[i] = w;
        if (i < rows) {
            store(i, w);
            if (tx == 0) s[(r0 + i) * sp + tc] = (uint8_t)rscale[i];
            if (tc == nbc - 1 && tx > 0 && tc + tx < sp) s[(r0 + i) * sp + tc + tx] = 127;
        }
    }
    if (!qt) return;
#pragma unroll
    for (int h = 0; h < 2; ++h) {   // columns 0 .. 3 and 4 .. 7 of the patch
        uint32_t up[4], down[4];
        auto half = [&](int i) { return h ? across[i].y : across[i].x; };
        turn4(half(0), half(1), half(2), half(3), up);
        turn4(half(4), half(5), half(6), half(7), down);
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<uint2 *>(&turned[place(tx * 8 + 4 * h + j, ty >> 1) + (ty & 1) * 8]) = make_uint2(up[j], down[j]);
    }
    if (ty == 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c0 + j < C) st[(c0 + j) * spt + tr] = (uint8_t)cscale[j];
    }
    if (tr == nbr - 1 && tr + ty < spt && ty > 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c0 + j < C) st[(c0 + j) * spt + tr + ty] = 127;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int piece = k * kThreads + threadIdx.x, col = piece / 8, part = piece & 7;
        const int64_t c = (int64_t)tc * 128 + col;
        if (c < C) *reinterpret_cast<uint4 *>(qt + c * nbr * 128 + (int64_t)tr * 128 + part * 16) = *reinterpret_cast<const uint4 *>(&turned[place(col, part)]);
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
    // the row copy alone: workgroups of 16 blocks, whole ones
    if (!square && !qt && rows * ((cols + 127) / 128) > most - 16) return Q8T_ERR_SHAPE;
    if (!x || !q || !s || !qt != !st) return Q8T_ERR_NULL;
    if (!q8t_aligned(q, 16) || (qt && !q8t_aligned(qt, 16))) return Q8T_ERR_SHAPE;
    const Args a = {x, rows, cols, seed, step, q, s, qt, st, (hipStream_t)stream};
    if (type == Q8T_F32)
        return format == Q8T_E4M3 ? choose<float, Q8T_E4M3>(a, square, stochastic) : choose<float, Q8T_E5M2>(a, square, stochastic);
    return format == Q8T_E4M3 ? choose<q8t_bf16, Q8T_E4M3>(a, square, stochastic) : choose<q8t_bf16, Q8T_E5M2>(a, square, stochastic);
}
