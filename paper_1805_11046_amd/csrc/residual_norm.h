// Kernels of the norms behind and in front of a block (residual_norm.hip has the entry points).  Per row of D:
//   m = h / rms(h)  (rms = sqrt(mean of squares + eps)),  u = m * w_post      (without w_post: u = h)
//   v = branch_scale * drop(gate * u),  r' = res_scale * r + v,  n = r' / rms(r'),  y = n * w_pre
// Backward, with dn = dy * w_pre and dm = du * w_post:
//   dr' = dres_out + (dn - n * mean(dn * n)) / rms(r'),   dr = res_scale * dr',   dv = branch_scale * drop(dr')
//   dgate = dv * u,  du = dv * gate,  dh = (dm - m * mean(dm * m)) / rms(h),  dw_pre = sum dy * n,  dw_post = sum du * m
// The mask is drawn again from (seed + step, flat position); 1 / rms of both norms is kept from the forward pass.
//
// Bound by memory: forward 4 tensors, backward 6, each crossing HBM once, so a row stays in registers between its passes: as many
// wavefronts as it takes hold it, eight or sixteen entries a thread, all sums in fp32, over those and then a tree.  What is close
// behind is the vector unit (some 26 operations an entry forward, ten of them for the mask), hence kernels for what the call has:
#pragma once
#include "fp8_codes.h"

// what a call has: a block output (else the norm in front is all), a norm behind the block, a gate, drop-out
struct NormCall {
    bool h, post, gate, drop;
};
struct Norm {
    const void *res, *h, *gate;
    const float *w_post, *w_pre;
    void *res_out, *y;
    float *stats;
    uint8_t *q, *s;
    int64_t T;
    int D;
    int64_t group_rows;   // rows that share a row of the gate
    float eps, res_scale, branch_scale;
    Q8tDrop d;
    uint64_t seed;
    const int64_t *step;
};
struct NormBack {
    const void *dy, *dres_out, *res_out, *h, *gate;
    const float *stats, *w_post, *w_pre;
    void *dres, *dh, *dgate;
    float *part;               // [chunks][sums][norm_part_width(D)]: dw_pre, dw_post, dgate, those that are wanted
    int sums, post_at, gate_at;   // place of dw_post and of dgate in a chunk's sums
    int64_t T;
    int D;
    int64_t group_rows, chunk_rows;   // rows of a chunk; a chunk holds whole groups or is part of one
    int64_t group_chunks;             // chunks of a group where that is split, else 0
    float res_scale, branch_scale;
    Q8tDrop d;
    uint64_t seed;
    const int64_t *step;
};

constexpr int kNormMaxD = 16384;

// Threads of a row: whole wavefronts, eight entries each, or sixteen where eight would take more than a workgroup has.
inline int norm_threads(int D)
{
    const int per = D <= 8192 ? 8 : 16;
    return ((D + per - 1) / per + 63) & ~63;
}

// entries of a row of partial sums: whole lines of 128 bytes
inline __host__ __device__ int norm_part_width(int D) { return (D + 31) & ~31; }

// residual_norm_{f32,bf16}.hip (forward) and residual_norm_bwd_{f32,bf16}.hip
void q8t_norm_fwd_f32(const Norm &a, const NormCall &c, hipStream_t st);
void q8t_norm_fwd_bf16(const Norm &a, const NormCall &c, hipStream_t st);
int q8t_norm_bwd_f32(const NormBack &a, const NormCall &c, int64_t chunks, hipStream_t st);
int q8t_norm_bwd_bf16(const NormBack &a, const NormCall &c, int64_t chunks, hipStream_t st);

namespace {

// MOST threads a row at most (up to 64: LANES of one wavefront, which has 64 / LANES rows at a time; else a workgroup), NV vectors of eight
// entries a thread; TINY: rows of fewer than eight.  A row's 16 lanes are the fewest, as many as hold a block of codes.
template <int MOST_, int NV_, bool TINY_>
struct NormShape {
    static constexpr int MOST = MOST_, NV = NV_, LANES = MOST < 64 ? MOST : 64, ROWS = 64 / LANES;
    static constexpr bool WAVE = MOST <= 64, TINY = TINY_;
};

// Sum over the threads of a row; every thread has it.  scratch: two sets of slots used in turn, so that one barrier a sum does.
template <class S>
__device__ __forceinline__ float row_sum(float v, float (*scratch)[16], int &turn)
{
#pragma unroll
    for (int off = S::LANES / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if (S::WAVE) return v;
    float *slot = scratch[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x / 64] = v;
    __syncthreads();
    const int waves = blockDim.x / 64;
    float t = 0.0f;
    for (int i = 0; i < waves; ++i) t += slot[i];
    return t;
}

// wavefronts of a SIMD that the registers have to allow, so that enough loads are in flight
template <class T, class S>
struct NormWaves {
    static constexpr bool SHORT = sizeof(T) == 2;
    static constexpr int FWD = S::NV == 1 && SHORT && S::ROWS == 1 ? 6 : 4, BWD = S::WAVE ? (SHORT && S::ROWS == 1 ? 4 : 3) : 4;
};

// Rows one after the other, a row's inputs asked for while the one before it is still worked on; the weights stay in registers.
// 8192 x 4096 bf16 with everything: 53 us, 5.1 TB/s, the rate of a copy; 6000 x 5120 53.5.
template <class T, class S, bool H, bool POST, bool GATE, bool DROP>
__global__ __launch_bounds__(S::WAVE ? 256 : S::MOST, (NormWaves<T, S>::FWD)) void norm_fwd(const Norm a)
{
    constexpr int NV = S::NV;
    constexpr bool WAVE = S::WAVE, TINY = S::TINY;
    __shared__ float scratch[2][16];
    int turn = 0;
    const uint32_t TH = WAVE ? 64 : blockDim.x, t = WAVE ? threadIdx.x & (S::LANES - 1) : threadIdx.x, D = a.D;
    const int64_t stride = WAVE ? (int64_t)gridDim.x * 4 * S::ROWS : gridDim.x;
    int64_t row = WAVE ? ((int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64)) * S::ROWS : blockIdx.x;
    if (S::ROWS > 1) row += threadIdx.x % 64 / S::LANES;
    if (row >= a.T) return;   // all threads of the row; a workgroup of several wavefronts has one
    const float rD = 1.0f / (float)D;
    const Q8tSeed sd = DROP ? q8t_seed(a.seed, a.step) : Q8tSeed{0, 0};
    const float scale = DROP ? a.branch_scale * a.d.scale : a.branch_scale;
    Q8tEight<T> xr[NV], xh[NV];
    float wpost[NV][8], wpre[NV][8];
    auto ask = [&](int64_t at) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            xr[j].template ask<TINY>((const T *)a.res + at * D, (j * TH + t) * 8, D);
            if (H) xh[j].template ask<TINY>((const T *)a.h + at * D, (j * TH + t) * 8, D);
        }
    };
    ask(row);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (POST) q8t_row8<TINY>(a.w_post, wpost[j], (j * TH + t) * 8, D);
        if (a.w_pre) q8t_row8<TINY>(a.w_pre, wpre[j], (j * TH + t) * 8, D);
    }
    for (; row < a.T; row += stride) {
        const int64_t base = row * D;
        float r[NV][8];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            xr[j].template settle<TINY>((j * TH + t) * 8, D);
            if (H) xh[j].template settle<TINY>((j * TH + t) * 8, D);
        }
        if (H) {
            float rstd = 1.0f;
            if (POST) {
                float ss = 0.0f;
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(xh[j][i], xh[j][i], ss);
#pragma unroll
                for (int j = 0; j < NV; ++j) xh[j].hold();
                rstd = 1.0f / __builtin_sqrtf(row_sum<S>(ss, scratch, turn) * rD + a.eps);
            }
            if (a.stats && t == 0) a.stats[row] = rstd;
            const float factor = rstd * scale;   // all that is the same for the row
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const uint32_t c = (j * TH + t) * 8;
                float u[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) u[i] = xh[j][i] * factor;
                if (POST) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[i] *= wpost[j][i];
                }
                if (GATE) {
                    float w[8];
                    q8t_row8<TINY>((const T *)a.gate + row / a.group_rows * D, w, c, D);
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[i] *= w[i];
                }
                if (DROP) {
                    uint32_t bits[4];
                    if (D % 4 == 0) q8t_draw8<true>(base + c, sd, bits);
                    else q8t_draw8<false>(base + c, sd, bits);
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[i] = q8t_kept(bits, i, a.d.below) ? u[i] : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) r[j][i] = __builtin_fmaf(xr[j][i], a.res_scale, u[i]);
                q8t_row_store8<true>((T *)a.res_out + base, c, r[j], D);
            }
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) r[j][i] = xr[j][i];
        }
        if (row + stride < a.T) ask(row + stride);
        if (!a.w_pre) continue;
        // y comes from the fp32 stream, not from what was rounded for res_out: one rounding instead of two
        float ss = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(r[j][i], r[j][i], ss);
        const float rstd = 1.0f / __builtin_sqrtf(row_sum<S>(ss, scratch, turn) * rD + a.eps);
        if (a.stats && t == 0) a.stats[a.T + row] = rstd;
        const uint32_t nb = (D + 127) / 128, sp = (nb + 3) & ~3u;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t c = (j * TH + t) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) r[j][i] = r[j][i] * rstd * wpre[j][i];
            if (a.y) q8t_row_store8<true>((T *)a.y + base, c, r[j], D);
            if (a.q) {
                if (D % 128) {   // behind the row's end the codes are zeros, also where 1 / rms is a NaN or infinite
#pragma unroll
                    for (int i = 0; i < 8; ++i) r[j][i] = c + i < D ? r[j][i] : 0.0f;
                }
                const uint32_t s = fp8_scale<Q8T_E4M3>(fp8_max16(fp8_max8(r[j])));   // 16 threads hold a block
                if (c < nb * 128) {
                    *reinterpret_cast<uint2 *>(a.q + row * nb * 128 + c) = fp8_codes8<Q8T_E4M3, false>(r[j], s, nullptr);
                    if (t % 16 == 0) a.s[row * sp + c / 128] = (uint8_t)s;
                }
            }
        }
        if (a.q && t < sp - nb) a.s[row * sp + nb + t] = 127;
    }
}

// rows [first, last) of chunk k
__device__ __forceinline__ void rows_of_chunk(const NormBack &a, int64_t k, int64_t &first, int64_t &last)
{
    if (a.group_chunks) {
        const int64_t g = k / a.group_chunks, part = k - g * a.group_chunks, start = g * a.group_rows;
        first = start + min(part * a.chunk_rows, a.group_rows);
        last = start + min((part + 1) * a.chunk_rows, a.group_rows);
    } else {
        first = k * a.chunk_rows;
        last = min(first + a.chunk_rows, a.T);
    }
}

// What a thread of the backward pass keeps in LDS, in places of its own (no barriers): eight entries a thread: the weights and a shared
// gate's row; sixteen: the sums over rows, for which registers have no room then.
struct LdsEights {
    float4 *base;
    uint32_t TH;
    __device__ __forceinline__ void load(int k, float v[8]) const
    {
        const float4 a = base[2 * k * TH], b = base[(2 * k + 1) * TH];
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
    __device__ __forceinline__ void store(int k, const float v[8])
    {
        base[2 * k * TH] = make_float4(v[0], v[1], v[2], v[3]);
        base[(2 * k + 1) * TH] = make_float4(v[4], v[5], v[6], v[7]);
    }
};
template <class S>
struct RowSums {   // over the rows of a chunk: of dw_pre, dw_post and a shared gate
    static constexpr int NV = S::NV, KEPT = NV == 1 ? 3 : 1;   // in registers: all, or the first
    float v[KEPT][NV][8];
    LdsEights lds;
    __device__ __forceinline__ void load(int k, int j, float s[8]) const
    {
        if (k < KEPT) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = v[k][j][i];
        } else {
            lds.load((k - KEPT) * NV + j, s);
        }
    }
    __device__ __forceinline__ void store(int k, int j, const float s[8])
    {
        if (k < KEPT) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][j][i] = s[i];
        } else {
            lds.store((k - KEPT) * NV + j, s);
        }
    }
    __device__ __forceinline__ void clear(int k)
    {
        const float zero[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < NV; ++j) store(k, j, zero);
    }
};
enum { SUM_PRE, SUM_POST, SUM_GATE };
template <class S>
constexpr int norm_bwd_lds()   // bytes a thread
{
    return (S::NV == 1 ? 3 : 2 * S::NV) * 32;
}

enum { GATE_NONE, GATE_SHARED, GATE_ROWS };   // a row of the gate for several rows, for each
// What a call of the backward pass has.  Known when compiled: both gradients, the norm in front and a block output, rows of eight entries at
// least.  Then no load or store hangs on a condition, and the compiler can count what is under way: a wait for one row's tensors does not
// become one for the next row's, which have just been asked for.  So every thread has eight whole entries: those behind the row's end do
// the last eight's work along with their owner; where D is no multiple of eight, the second thread's begin among the first one's, and the
// sums over the row leave out what is another's.  Such threads are in one wavefront, so that dres may lie where dy or dres_out does; with
// two vectors a thread some are not, and such a call takes the other form.
// Both passes over the rows and the sums, 6000 x 5120 bf16, us, with 512 chunks: conditional 125, known 94.
template <bool POST, int GATE, bool DROP, bool EVEN>
struct BackKnown {
    static constexpr bool h = true, pre = true, out = true, post = POST, drop = DROP, known = true, even = EVEN;
    static constexpr int gate = GATE;
    __device__ explicit BackKnown(const NormBack &) {}
};
struct BackAsked {
    static constexpr bool known = false, even = false;
    bool h, pre, out, post, drop;
    int gate;
    __device__ explicit BackAsked(const NormBack &a)
        : h(a.h), pre(a.w_pre), out(a.dres_out), post(a.w_post), drop(a.d.cut != 0), gate(!a.gate ? GATE_NONE : (a.group_rows > 1 ? GATE_SHARED : GATE_ROWS))
    {
    }
};

// One workgroup a chunk of rows: the column sums go to the workspace once; the tensors of the next row are asked for as soon as this
// row's have been used, into the same registers (sixteen entries a thread leave no room for that: they are asked for where the row begins,
// 1000 x 16384 bf16 114 us for 150 with 512 chunks).  Bound by memory: 6000 x 5120 bf16 with a shared gate
// and drop-out 86 us, 369 MB and 15 MB of partial sums at 4.5 TB/s; 8192 x 4096 at 4.8 TB/s.
template <class T, class S, class F>
__global__ __launch_bounds__(S::WAVE ? 64 : S::MOST, (NormWaves<T, S>::BWD)) void norm_bwd(const NormBack a)
{
    constexpr int NV = S::NV;
    constexpr bool WAVE = S::WAVE, TINY = S::TINY, KNOWN = F::known, WEIGHTS_KEPT = NV == 1, AHEAD = NV == 1;
    extern __shared__ float4 kept[];
    __shared__ float scratch[2][16];
    int turn = 0;
    const F f(a);
    const uint32_t t = WAVE ? threadIdx.x & (S::LANES - 1) : threadIdx.x, D = a.D, TH = WAVE ? 64 : blockDim.x;
    const float rD = 1.0f / (float)D;
    int64_t first, last;
    rows_of_chunk(a, blockIdx.x, first, last);
    if (S::ROWS > 1) {   // a part of the chunk for each row that the wavefront has at a time, of whole groups where the chunk is
        const int64_t unit = f.gate == GATE_SHARED && !a.group_chunks ? a.group_rows : 1;
        const int64_t rows = ((last - first) / unit + S::ROWS - 1) / S::ROWS * unit;
        first = min(first + (int64_t)(threadIdx.x / S::LANES) * rows, last);
        last = min(first + rows, last);
    }
    const Q8tSeed sd = f.drop ? q8t_seed(a.seed, a.step) : Q8tSeed{0, 0};
    const float scale = f.drop ? a.branch_scale * a.d.scale : a.branch_scale;
    const LdsEights lds = {kept + threadIdx.x, TH};
    RowSums<S> sums;
    sums.lds = lds;
#pragma unroll
    for (int k = 0; k < 3; ++k) sums.clear(k);

    const uint32_t eights = (D + 7) / 8, shared = eights * 8 - D;
    auto col = [&](int j) -> uint32_t {   // the first of a thread's eight entries
        const uint32_t k = j * TH + t;
        if (!KNOWN) return k * 8;
        return min(!F::even && k ? k * 8 - shared : k * 8, D - 8);
    };
    auto others = [&](int j) -> int {   // how many of them, from the first on, are another thread's
        const uint32_t k = j * TH + t;
        return k >= eights ? 8 : (!F::even && k == 1 ? (int)shared : 0);
    };
    auto add = [&](float &dot, const float a[8], const float b[8], int j) {   // dot += a . b over the thread's own
        float d = 0.0f;
        const int from = KNOWN ? others(j) : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) d = __builtin_fmaf(!KNOWN || F::even || i >= from ? a[i] : 0.0f, b[i], d);
        dot += !KNOWN || !F::even || from == 0 ? d : 0.0f;
    };
    auto ask8 = [&](Q8tEight<T> &x, const T *row, int j) {
        if (KNOWN) x.template vector<true>(q8t_at(row, col(j)));
        else x.template ask<TINY>(row, col(j), D);
    };
    auto settle = [&](Q8tEight<T> &x, int j) {
        if (!KNOWN) x.template settle<TINY>(col(j), D);
    };
    auto put = [&](T *row, int j, const float v[8]) {
        if (KNOWN) q8t_store8<false>(q8t_at(row, col(j)), v);
        else q8t_row_store8(row, col(j), v, D);
    };
    auto gate_row = [&](int64_t g) { return (const T *)a.gate + g * D; };
    auto keep = [&](int k, auto row) {
        float w[8];
        q8t_row8<TINY>(row, w, col(0), D);
        const_cast<LdsEights &>(lds).store(k, w);
    };
    int64_t group = f.gate == GATE_SHARED ? first / a.group_rows : 0, group_end = f.gate == GATE_SHARED ? (group + 1) * a.group_rows : 0;
    if (WEIGHTS_KEPT && first < last) {
        if (f.pre) keep(SUM_PRE, a.w_pre);
        if (f.post) keep(SUM_POST, a.w_post);
        if (f.gate == GATE_SHARED) keep(SUM_GATE, gate_row(group));
    }
    auto weights = [&](int k, float w[8], auto row, int j) {
        if (WEIGHTS_KEPT) lds.load(k, w);
        else q8t_row8<TINY>(row, w, col(j), D);
    };

    Q8tEight<T> xdy[NV], xout[NV], xr[NV], xh[NV], xg[NV];
    float rstd_pre = 0.0f, rstd_post = 1.0f;
    auto ask = [&](int64_t row) {
        if (f.pre) rstd_pre = a.stats[a.T + row];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (f.pre) {
                ask8(xdy[j], (const T *)a.dy + row * D, j);
                ask8(xr[j], (const T *)a.res_out + row * D, j);
            }
            if (f.out) ask8(xout[j], (const T *)a.dres_out + row * D, j);
        }
    };
    auto ask_h = [&](int64_t row) {
        if (f.post) rstd_post = a.stats[row];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            ask8(xh[j], (const T *)a.h + row * D, j);
            if (f.gate == GATE_ROWS) ask8(xg[j], gate_row(row), j);
        }
    };
    if (AHEAD && first < last) {
        ask(first);
        if (f.h) ask_h(first);
    }
    for (int64_t row = first; row < last; ++row) {
        const int64_t base = row * D, after = min(row + 1, last - 1);   // behind the last row that one again
        float dr[NV][8], dot = 0.0f;
        if (!AHEAD) ask(row);
        if (f.pre) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                settle(xdy[j], j);
                settle(xr[j], j);
                float w[8], s[8], n[8];
                weights(SUM_PRE, w, a.w_pre, j);
                sums.load(SUM_PRE, j, s);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    n[i] = xr[j][i] * rstd_pre;
                    s[i] = __builtin_fmaf(xdy[j][i], n[i], s[i]);
                    dr[j][i] = xdy[j][i] * w[i];
                }
                add(dot, dr[j], n, j);
                sums.store(SUM_PRE, j, s);
                xr[j].hold();
            }
            const float mean = row_sum<S>(dot, scratch, turn) * rD, k = rstd_pre * rstd_pre * mean;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) dr[j][i] = __builtin_fmaf(dr[j][i], rstd_pre, -(xr[j][i] * k));
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) dr[j][i] = 0.0f;
        }
        if (f.out) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                settle(xout[j], j);
#pragma unroll
                for (int i = 0; i < 8; ++i) dr[j][i] += xout[j][i];
            }
        }
        if (AHEAD) ask(after);
        else if (f.h) ask_h(row);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = dr[j][i] * a.res_scale;
            put((T *)a.dres + base, j, o);
        }
        if (!f.h) continue;
        if (f.gate == GATE_SHARED && row >= group_end) {
            ++group;
            group_end += a.group_rows;
            if (WEIGHTS_KEPT) keep(SUM_GATE, gate_row(group));
        }
        dot = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            settle(xh[j], j);
            // A position that is not kept takes nothing of h and the gate, and gives nothing to their gradients: left out of what is read with
            // two vectors a thread, else of the products (fp32 1000 x 16384 219 and 238 us, 8192 x 4096 207 and 196).
            constexpr bool EARLY = NV > 1;
            bool kept[8];
            auto counts = [&](int i) { return EARLY || !f.drop || kept[i]; };
            if (f.drop) {
                uint32_t bits[4];
                if (D % 4 == 0) q8t_draw8<true>(base + col(j), sd, bits);
                else q8t_draw8<false>(base + col(j), sd, bits);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    kept[i] = q8t_kept(bits, i, a.d.below);
                    dr[j][i] = kept[i] ? dr[j][i] * scale : 0.0f;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) dr[j][i] *= scale;
            }
            float w[8];
            if (f.post) weights(SUM_POST, w, a.w_post, j);
            if (f.gate != GATE_NONE) {
                float g[8], o[8], s[8];
                if (f.gate == GATE_SHARED) {
                    weights(SUM_GATE, g, gate_row(group), j);
                } else {
                    settle(xg[j], j);
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[i] = xg[j][i];
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float m = xh[j][i] * rstd_post;
                    o[i] = f.post ? m * w[i] : m;
                    if (EARLY && f.drop) {
                        o[i] = kept[i] ? o[i] : 0.0f;
                        g[i] = kept[i] ? g[i] : 0.0f;
                    }
                }
                if (f.gate == GATE_SHARED) {
                    sums.load(SUM_GATE, j, s);
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[i] = counts(i) ? __builtin_fmaf(dr[j][i], o[i], s[i]) : s[i];
                    sums.store(SUM_GATE, j, s);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[i] = counts(i) ? o[i] * dr[j][i] : 0.0f;
                    put((T *)a.dgate + base, j, o);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) dr[j][i] *= counts(i) ? g[i] : 0.0f;
            }
            if (f.post) {
                float s[8], m[8];
                sums.load(SUM_POST, j, s);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    m[i] = xh[j][i] * rstd_post;
                    s[i] = __builtin_fmaf(dr[j][i], m[i], s[i]);
                    dr[j][i] *= w[i];
                }
                add(dot, dr[j], m, j);
                sums.store(SUM_POST, j, s);
            }
            xh[j].hold();
        }
        float k = 0.0f;
        if (f.post) k = rstd_post * rstd_post * (row_sum<S>(dot, scratch, turn) * rD);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (f.post) {
#pragma unroll
                for (int i = 0; i < 8; ++i) dr[j][i] = __builtin_fmaf(dr[j][i], rstd_post, -(xh[j][i] * k));
            }
            put((T *)a.dh + base, j, dr[j]);
        }
        if (AHEAD) ask_h(after);
        if (f.gate == GATE_SHARED && !a.group_chunks && row + 1 == group_end) {   // a whole group inside the chunk
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float s[8];
                sums.load(SUM_GATE, j, s);
                put((T *)a.dgate + group * D, j, s);
            }
            sums.clear(SUM_GATE);
        }
    }
    if (S::ROWS > 1) {
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            float s[8];
            sums.load(k, 0, s);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
#pragma unroll
                for (int off = S::LANES; off < 64; off *= 2) s[i] += __shfl_xor(s[i], off, 64);
            }
            sums.store(k, 0, s);
        }
        if (threadIdx.x >= S::LANES) return;
    }
    float *part = a.part + (int64_t)blockIdx.x * a.sums * norm_part_width(D);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const uint32_t c = col(j);
        float s[8];
        if (f.pre) {
            sums.load(SUM_PRE, j, s);
            q8t_row_store8(part, c, s, D);
        }
        if (f.post) {
            sums.load(SUM_POST, j, s);
            q8t_row_store8(part + (int64_t)a.post_at * norm_part_width(D), c, s, D);
        }
        if (f.gate == GATE_SHARED && a.gate_at >= 0) {
            sums.load(SUM_GATE, j, s);
            q8t_row_store8(part + (int64_t)a.gate_at * norm_part_width(D), c, s, D);
        }
    }
}

// run(shape) with the row's shape as a type
template <class R>
void norm_by_width(int D, R run)
{
    // 100000 x 64 bf16, us, one row or four a wavefront: forward 70 and 26, backward 89 and 38
    if (D < 8) run(NormShape<16, 1, true>());
    else if (D <= 128) run(NormShape<16, 1, false>());
    else if (D <= 256) run(NormShape<32, 1, false>());
    else if (D <= 512) run(NormShape<64, 1, false>());
    else if (D <= 8192) run(NormShape<1024, 1, false>());
    else run(NormShape<1024, 2, false>());
}

template <class T>
void run_norm_fwd(const Norm &a, const NormCall &c, hipStream_t st)
{
    typedef std::true_type Y;
    typedef std::false_type N;
    norm_by_width(a.D, [&](auto shape) {
        typedef decltype(shape) S;
        // as many workgroups as the chip holds at 24 wavefronts a compute unit (16 where a thread has two vectors); each takes rows one
        // after the other
        const int threads = S::WAVE ? 256 : norm_threads(a.D);
        const int64_t groups = S::WAVE ? (a.T + 4 * S::ROWS - 1) / (4 * S::ROWS) : a.T, most = 256 * ((S::NV == 1 ? 24 : 16) * 64 / threads);
        const unsigned grid = (unsigned)(groups < most ? groups : most);
        auto launch = [&](auto h, auto post, auto gate, auto drop) {
            norm_fwd<T, S, decltype(h)::value, decltype(post)::value, decltype(gate)::value, decltype(drop)::value><<<grid, threads, 0, st>>>(a);
        };
        auto drop = [&](auto post, auto gate) { c.drop ? launch(Y(), post, gate, Y()) : launch(Y(), post, gate, N()); };
        if (!c.h) launch(N(), N(), N(), N());
        else if (c.post) c.gate ? drop(Y(), Y()) : drop(Y(), N());
        else c.gate ? drop(N(), Y()) : drop(N(), N());
    });
}

template <class T, class S, class F>
int launch_norm_bwd(const NormBack &a, int64_t chunks, hipStream_t st)
{
    constexpr int BYTES = norm_bwd_lds<S>();
    const auto kernel = norm_bwd<T, S, F>;
    static Q8tLdsOptIn opt;
    if (BYTES * S::MOST > 60 * 1024) {
        const int rc = q8t_allow_lds(opt, (const void *)kernel, BYTES * S::MOST);
        if (rc) return rc;
    }
    const int threads = norm_threads(a.D);
    kernel<<<(unsigned)chunks, threads, BYTES * threads, st>>>(a);
    return Q8T_OK;
}
template <class T>
int run_norm_bwd(const NormBack &a, const NormCall &c, int64_t chunks, hipStream_t st)
{
    int rc = Q8T_OK;
    norm_by_width(a.D, [&](auto shape) {
        typedef decltype(shape) S;
        // fp32 with all three sums over the rows: what the known form keeps under way does not fit 128 registers (8192 x 4096 236 us, asked 189;
        // 6000 x 5119 290 and 236; 32768 x 768 199 and 146)
        constexpr bool CROWDED = sizeof(T) == 4 && !S::WAVE;
        const bool over = S::NV > 1 && (a.dres == a.dy || a.dres == a.dres_out);
        if (over || (CROWDED && c.post && c.gate && a.group_rows > 1) || S::TINY || !c.h || !a.w_pre || !a.dres_out) {
            rc = launch_norm_bwd<T, S, BackAsked>(a, chunks, st);
            return;
        }
        if constexpr (!S::TINY) {
            auto drop = [&](auto post, auto gate) {
                constexpr bool P = decltype(post)::value;
                constexpr int G = decltype(gate)::value;
                auto even = [&](auto drops) {
                    constexpr bool K = decltype(drops)::value;
                    if constexpr (!CROWDED || !P || G != GATE_SHARED) rc = a.D % 8 ? launch_norm_bwd<T, S, BackKnown<P, G, K, false>>(a, chunks, st) : launch_norm_bwd<T, S, BackKnown<P, G, K, true>>(a, chunks, st);
                };
                c.drop ? even(std::true_type()) : even(std::false_type());
            };
            auto gate = [&](auto post) {
                if (!c.gate) drop(post, std::integral_constant<int, GATE_NONE>());
                else if (a.group_rows > 1) drop(post, std::integral_constant<int, GATE_SHARED>());
                else drop(post, std::integral_constant<int, GATE_ROWS>());
            };
            c.post ? gate(std::true_type()) : gate(std::false_type());
        }
    });
    return rc;
}

}  // namespace
