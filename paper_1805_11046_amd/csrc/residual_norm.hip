// The end of one transformer block and the start of the next in one pass over the rows of the residual stream.  Per row of D:
//   m = h / rms(h)  (rms = sqrt(mean of squares + eps)),  u = m * w_post      (without w_post: u = h)
//   v = branch_scale * drop(gate * u),  r' = res_scale * r + v,  n = r' / rms(r'),  y = n * w_pre
// Backward, with dn = dy * w_pre and dm = du * w_post:
//   dr' = dres_out + (dn - n * mean(dn * n)) / rms(r'),   dr = res_scale * dr',   dv = branch_scale * drop(dr')
//   dgate = dv * u,  du = dv * gate,  dh = (dm - m * mean(dm * m)) / rms(h),  dw_pre = sum dy * n,  dw_post = sum du * m
// The mask is drawn again from (seed + step, flat position); 1 / rms of both norms is kept from the forward pass.
//
// Bound by memory: forward 4 tensors, backward 6, each crossing HBM once, so a row stays in registers between its passes: TH
// threads hold it, 8 * NV entries each, all sums in fp32 over at most 64 terms a thread and then a tree.
#include "fp8_codes.h"

namespace {

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
    bool drop;
    Q8tDrop d;
    uint64_t seed;
    const int64_t *step;
};

// sum over the TH threads of a row; every thread has it.  `scratch`: two sets of slots used in turn, so that one barrier a sum does
template <int TH>
__device__ __forceinline__ float row_sum(float v, float (*scratch)[16], int &turn)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if (TH == 64) return v;
    constexpr int W = TH / 64;
    float *slot = scratch[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x / 64] = v;
    __syncthreads();
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) t += slot[i];
    return t;
}

template <class T, int TH, int NV, bool DROP, bool ALIGNED>
__global__ __launch_bounds__(TH < 256 ? 256 : TH) void norm_fwd(const Norm a)
{
    __shared__ float scratch[2][16];
    constexpr int ROWS = TH < 256 ? 256 / TH : 1;
    int turn = 0;
    const int t = threadIdx.x % TH;
    const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TH;
    if (row >= a.T) return;   // whole wavefronts; with more than one a row there is one row a workgroup
    const int D = a.D;
    const int64_t base = row * D;
    const float rD = 1.0f / (float)D;
    float r[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) q8t_load8((const T *)a.res + base + (j * TH + t) * 8, r[j], D - (j * TH + t) * 8);
    if (a.h) {
        float u[NV][8];
#pragma unroll
        for (int j = 0; j < NV; ++j) q8t_load8((const T *)a.h + base + (j * TH + t) * 8, u[j], D - (j * TH + t) * 8);
        float rstd = 1.0f;
        if (a.w_post) {
            float ss = 0.0f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) ss += u[j][i] * u[j][i];
            rstd = 1.0f / __builtin_sqrtf(row_sum<TH>(ss, scratch, turn) * rD + a.eps);
        }
        if (a.stats && t == 0) a.stats[row] = rstd;
        const Q8tSeed sd = DROP ? q8t_seed(a.seed, a.step) : Q8tSeed{0, 0};
        const float scale = DROP ? a.branch_scale * a.d.scale : a.branch_scale;
        const T *gate = (const T *)a.gate;
        if (gate) gate += row / a.group_rows * D;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TH + t) * 8, count = D - c;
            float w[8];
            if (a.w_post) {
                q8t_load8_kept(a.w_post + c, w, count);
#pragma unroll
                for (int i = 0; i < 8; ++i) u[j][i] = u[j][i] * rstd * w[i];
            }
            if (gate) {
                q8t_load8_kept(gate + c, w, count);
#pragma unroll
                for (int i = 0; i < 8; ++i) u[j][i] *= w[i];
            }
            if (DROP) {
                uint32_t bits[8];
                q8t_draw8<ALIGNED>(base + c, sd, bits);
#pragma unroll
                for (int i = 0; i < 8; ++i) u[j][i] = bits[i] >= a.d.cut ? u[j][i] * scale : 0.0f;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) u[j][i] *= scale;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) r[j][i] = r[j][i] * a.res_scale + u[j][i];
            q8t_store8((T *)a.res_out + base + c, r[j], count);
        }
    }
    if (!a.w_pre) return;
    // y comes from the fp32 stream, not from what was rounded for res_out: one rounding instead of two
    float ss = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += r[j][i] * r[j][i];
    const float rstd = 1.0f / __builtin_sqrtf(row_sum<TH>(ss, scratch, turn) * rD + a.eps);
    if (a.stats && t == 0) a.stats[a.T + row] = rstd;
    const int nb = (D + 127) / 128, sp = (nb + 3) & ~3;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * TH + t) * 8, count = D - c;
        float w[8];
        q8t_load8_kept(a.w_pre + c, w, count);
#pragma unroll
        for (int i = 0; i < 8; ++i) r[j][i] = r[j][i] * rstd * w[i];
        if (a.y) q8t_store8((T *)a.y + base + c, r[j], count);
        if (a.q) {
            const uint32_t scale = fp8_scale<Q8T_E4M3>(fp8_max16(fp8_max8(r[j])));   // 16 threads hold a block
            if (c < nb * 128) {
                *reinterpret_cast<uint2 *>(a.q + row * nb * 128 + c) = fp8_codes8<Q8T_E4M3, false>(r[j], scale, nullptr);
                if (t % 16 == 0) a.s[row * sp + c / 128] = (uint8_t)scale;
            }
        }
    }
    if (a.q && t < sp - nb) a.s[row * sp + nb + t] = 127;
}

struct NormBack {
    const void *dy, *dres_out, *res_out, *h, *gate;
    const float *stats, *w_post, *w_pre;
    void *dres, *dh, *dgate;
    float *part;               // [chunks][sums][D]: dw_pre, dw_post, dgate, those that are wanted
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

// One workgroup a chunk of rows: the column sums stay in registers from row to row and go to the workspace once.
template <class T, int TH, int NV, bool DROP, bool ALIGNED>
__global__ __launch_bounds__(TH) void norm_bwd(const NormBack a)
{
    __shared__ float scratch[2][16];
    int turn = 0;
    const int t = threadIdx.x, D = a.D;
    const float rD = 1.0f / (float)D;
    int64_t first, last;
    rows_of_chunk(a, blockIdx.x, first, last);
    const Q8tSeed sd = DROP ? q8t_seed(a.seed, a.step) : Q8tSeed{0, 0};
    const float scale = DROP ? a.branch_scale * a.d.scale : a.branch_scale;
    const bool gated = a.gate && a.h, shared_gate = gated && a.group_rows > 1;
    float spre[NV][8], spost[NV][8], sgate[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) spre[j][i] = spost[j][i] = sgate[j][i] = 0.0f;
    int64_t group = gated ? first / a.group_rows : 0, group_end = gated ? (group + 1) * a.group_rows : 0;
    for (int64_t row = first; row < last; ++row) {
        const int64_t base = row * D;
        float dr[NV][8];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TH + t) * 8;
            if (a.dres_out) {
                q8t_load8((const T *)a.dres_out + base + c, dr[j], D - c);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) dr[j][i] = 0.0f;
            }
        }
        if (a.w_pre) {
            const float rstd = a.stats[a.T + row];
            float n[NV][8], dn[NV][8], dot = 0.0f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * TH + t) * 8;
                q8t_load8((const T *)a.res_out + base + c, n[j], D - c);
                q8t_load8((const T *)a.dy + base + c, dn[j], D - c);
            }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * TH + t) * 8;
                float w[8];
                q8t_load8_kept(a.w_pre + c, w, D - c);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    n[j][i] *= rstd;
                    spre[j][i] += dn[j][i] * n[j][i];
                    dn[j][i] *= w[i];
                    dot += dn[j][i] * n[j][i];
                }
            }
            const float mean = row_sum<TH>(dot, scratch, turn) * rD;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) dr[j][i] += rstd * (dn[j][i] - n[j][i] * mean);
        }
        if (a.dres) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * TH + t) * 8;
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = dr[j][i] * a.res_scale;
                q8t_store8((T *)a.dres + base + c, o, D - c);
            }
        }
        if (!a.h) continue;
        if (gated && row >= group_end) {
            ++group;
            group_end += a.group_rows;
        }
        const float rstd = a.w_post ? a.stats[row] : 1.0f;
        float m[NV][8], dot = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TH + t) * 8, count = D - c;
            q8t_load8((const T *)a.h + base + c, m[j], count);
            if (DROP) {
                uint32_t bits[8];
                q8t_draw8<ALIGNED>(base + c, sd, bits);
#pragma unroll
                for (int i = 0; i < 8; ++i) dr[j][i] = bits[i] >= a.d.cut ? dr[j][i] * scale : 0.0f;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) dr[j][i] *= scale;
            }
            float w[8];
            if (a.w_post) q8t_load8_kept(a.w_post + c, w, count);
#pragma unroll
            for (int i = 0; i < 8; ++i) m[j][i] *= rstd;
            if (gated) {
                float g[8], o[8];
                q8t_load8_kept((const T *)a.gate + group * D + c, g, count);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    o[i] = dr[j][i] * (a.w_post ? m[j][i] * w[i] : m[j][i]);
                    sgate[j][i] += o[i];
                    dr[j][i] *= g[i];
                }
                if (!shared_gate) q8t_store8((T *)a.dgate + base + c, o, count);
            }
            if (a.w_post) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    spost[j][i] += dr[j][i] * m[j][i];
                    dr[j][i] *= w[i];
                    dot += dr[j][i] * m[j][i];
                }
            }
        }
        float mean = 0.0f;
        if (a.w_post) mean = row_sum<TH>(dot, scratch, turn) * rD;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TH + t) * 8;
            if (a.w_post) {
#pragma unroll
                for (int i = 0; i < 8; ++i) dr[j][i] = rstd * (dr[j][i] - m[j][i] * mean);
            }
            q8t_store8((T *)a.dh + base + c, dr[j], D - c);
        }
        if (shared_gate && !a.group_chunks && row + 1 == group_end) {   // a whole group inside the chunk
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = (j * TH + t) * 8;
                q8t_store8((T *)a.dgate + group * D + c, sgate[j], D - c);
#pragma unroll
                for (int i = 0; i < 8; ++i) sgate[j][i] = 0.0f;
            }
        }
    }
    float *part = a.part + (int64_t)blockIdx.x * a.sums * D;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * TH + t) * 8;
        if (a.w_pre) q8t_store8(part + c, spre[j], D - c);
        if (a.post_at >= 0) q8t_store8(part + (int64_t)a.post_at * D + c, spost[j], D - c);
        if (a.gate_at >= 0) q8t_store8(part + (int64_t)a.gate_at * D + c, sgate[j], D - c);
    }
}

// Column sums of the chunks' partial sums, in one order whatever the launch: 16 columns x 16 threads, each over every 16th chunk.
// z = 0: dw_pre, 1: dw_post (over all chunks), from 2 on: one group of the gate.
template <class T>
__global__ __launch_bounds__(256) void norm_bwd_columns(const float *__restrict__ part, int sums, int post_at, int gate_at, int D,
                                                        int64_t chunks, int64_t group_chunks, bool pre, float *dw_pre, float *dw_post,
                                                        T *dgate)
{
    __shared__ float fold[16][17];
    const int tx = threadIdx.x & 15, ty = threadIdx.x / 16, c = blockIdx.x * 16 + tx;
    int64_t z = blockIdx.y, first = 0, count = chunks;
    int at = 0;
    const int weights = (pre ? 1 : 0) + (post_at >= 0 ? 1 : 0);
    if (z >= weights) {
        first = (z - weights) * group_chunks;
        count = group_chunks;
        at = gate_at;
    } else if (!pre || z == 1) {
        at = post_at;
    }
    float v = 0.0f;
    if (c < D)
        for (int64_t k = ty; k < count; k += 16) v += part[((first + k) * sums + at) * D + c];
    fold[ty][tx] = v;
    __syncthreads();
    if (ty || c >= D) return;
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += fold[i][tx];
    if (z >= weights) dgate[(z - weights) * D + c] = (T)v;
    else (at == post_at ? dw_post : dw_pre)[c] = v;
}

template <class T>
__global__ __launch_bounds__(256) void clear(T *p, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = (T)0.0f;
}

constexpr int kMaxD = 16384, kChunks = 512;

// threads of a row and vectors of eight a thread
struct Shape {
    int th, nv;
};
Shape shape_of(int D)
{
    if (D <= 512) return {64, 1};
    if (D <= 2048) return {256, 1};
    if (D <= 4096) return {512, 1};
    if (D <= 8192) return {1024, 1};
    return {1024, 2};
}

// Rows of a chunk of the backward pass.  Groups shorter than a chunk are taken whole (their gate's gradient is final there),
// longer ones are cut.
struct Chunks {
    int64_t rows, per_group, count;
};
Chunks chunks_of(int64_t T, int64_t group_rows)
{
    int64_t rows = (T + kChunks - 1) / kChunks;
    if (group_rows <= rows) {
        rows = (rows + group_rows - 1) / group_rows * group_rows;
        return {rows, 0, (T + rows - 1) / rows};
    }
    const int64_t per = (group_rows + rows - 1) / rows;   // at least two; fewer than kChunks groups are cut
    return {(group_rows + per - 1) / per, per, per * (T / group_rows)};
}

int check(int type, int64_t T, int D, int64_t groups, double p, Q8tDrop *d)
{
    if (T < 0 || D < 1 || D > kMaxD || groups < 0 || (groups > 0 && T % groups)) return Q8T_ERR_SHAPE;
    if (T > ((int64_t)1 << 34) / D || T >= (int64_t)1 << 22) return Q8T_ERR_SHAPE;
    if ((type != Q8T_F32 && type != Q8T_BF16) || !q8t_drop(p, d)) return Q8T_ERR_VALUE;
    return Q8T_OK;
}

template <class T, int TH, int NV>
void run_fwd(const Norm &a, hipStream_t st)
{
    constexpr int ROWS = TH < 256 ? 256 / TH : 1;
    const dim3 grid((unsigned)((a.T + ROWS - 1) / ROWS)), block(TH < 256 ? 256 : TH);
    if (!a.drop) norm_fwd<T, TH, NV, false, true><<<grid, block, 0, st>>>(a);
    else if (a.D % 4 == 0) norm_fwd<T, TH, NV, true, true><<<grid, block, 0, st>>>(a);
    else norm_fwd<T, TH, NV, true, false><<<grid, block, 0, st>>>(a);
}
template <class T, int TH, int NV>
void run_bwd(const NormBack &a, int64_t chunks, bool drop, hipStream_t st)
{
    const dim3 grid((unsigned)chunks), block(TH);
    if (!drop) norm_bwd<T, TH, NV, false, true><<<grid, block, 0, st>>>(a);
    else if (a.D % 4 == 0) norm_bwd<T, TH, NV, true, true><<<grid, block, 0, st>>>(a);
    else norm_bwd<T, TH, NV, true, false><<<grid, block, 0, st>>>(a);
}
#define Q8T_BY_SHAPE(f, T, D, ...)                                       \
    do {                                                                 \
        const Shape w = shape_of(D);                                     \
        if (w.th == 64) f<T, 64, 1>(__VA_ARGS__);                        \
        else if (w.th == 256) f<T, 256, 1>(__VA_ARGS__);                 \
        else if (w.th == 512) f<T, 512, 1>(__VA_ARGS__);                 \
        else if (w.nv == 1) f<T, 1024, 1>(__VA_ARGS__);                  \
        else f<T, 1024, 2>(__VA_ARGS__);                                 \
    } while (0)

}  // namespace

extern "C" {

int q8t_residual_norm_fwd(const void *res, const void *h, const float *w_post, const void *gate, int64_t groups, const float *w_pre, int type,
                          int64_t T, int D, float eps, float res_scale, float branch_scale, double p, uint64_t seed, const int64_t *step,
                          void *res_out, void *y, float *stats, uint8_t *q, uint8_t *s, void *stream)
{
    Q8tDrop d;
    const int rc = check(type, T, D, groups, p, &d);
    if (rc) return rc;
    if (T == 0) return Q8T_OK;
    if (!h && (w_post || gate || d.cut || res_scale != 1.0f)) return Q8T_ERR_VALUE;
    if ((gate != nullptr) != (groups > 0)) return Q8T_ERR_SHAPE;
    if (!res || (h && !res_out) || (!h && !w_pre) || !q != !s || (w_pre && !y && !q) || (!w_pre && (y || q))) return Q8T_ERR_NULL;
    if (q && !q8t_aligned(q, 16)) return Q8T_ERR_SHAPE;
    const Norm a = {res, h, gate, w_post, w_pre, res_out, y, stats, q, s, T, D, groups ? T / groups : 1, eps, res_scale, branch_scale,
                    d.cut != 0, d, seed, step};
    hipStream_t st = (hipStream_t)stream;
    if (type == Q8T_F32) Q8T_BY_SHAPE(run_fwd, float, D, a, st);
    else Q8T_BY_SHAPE(run_fwd, q8t_bf16, D, a, st);
    Q8T_LAUNCH_CHECK();
    return Q8T_OK;
}

size_t q8t_residual_norm_bwd_workspace_size(int64_t T, int D, int64_t groups)
{
    if (T <= 0 || D < 1 || D > kMaxD || groups < 0 || (groups > 0 && T % groups) || T >= (int64_t)1 << 22) return 0;
    return (size_t)chunks_of(T, groups ? T / groups : 1).count * 3 * D * sizeof(float);
}

int q8t_residual_norm_bwd(const void *dy, const void *dres_out, const void *res_out, const void *h, const float *stats, const float *w_post,
                          const void *gate, int64_t groups, const float *w_pre, int type, int64_t T, int D, float res_scale,
                          float branch_scale, double p, uint64_t seed, const int64_t *step, void *dres, void *dh, void *dgate,
                          float *dw_post, float *dw_pre, void *ws, void *stream)
{
    Q8tDrop d;
    const int rc = check(type, T, D, groups, p, &d);
    if (rc) return rc;
    hipStream_t st = (hipStream_t)stream;
    if (T == 0) {   // no rows: the sums over them are zero (tensors without entries may come without an address)
        const int64_t n = dgate ? groups * D : 0;
        const unsigned few = (unsigned)(n < 1 << 20 ? (n + 255) / 256 : 4096);
        if (dw_pre) clear<<<(D + 255) / 256, 256, 0, st>>>(dw_pre, D);
        if (dw_post) clear<<<(D + 255) / 256, 256, 0, st>>>(dw_post, D);
        if (n && type == Q8T_F32) clear<<<few, 256, 0, st>>>((float *)dgate, n);
        if (n && type == Q8T_BF16) clear<<<few, 256, 0, st>>>((q8t_bf16 *)dgate, n);
        Q8T_LAUNCH_CHECK();
        return Q8T_OK;
    }
    if (!h && (w_post || gate || d.cut || res_scale != 1.0f)) return Q8T_ERR_VALUE;
    if ((gate != nullptr) != (groups > 0)) return Q8T_ERR_SHAPE;
    if (!w_pre != !dy || !w_pre != !dw_pre || !w_post != !dw_post || !gate != !dgate || !h != !dh || (!dy && !dres_out)) return Q8T_ERR_NULL;
    if ((w_pre && !res_out) || ((w_pre || w_post) && !stats) || (!dres && !h)) return Q8T_ERR_NULL;
    const int64_t group_rows = groups ? T / groups : 1;
    const Chunks k = chunks_of(T, group_rows);
    const bool gate_parts = gate && k.per_group;
    if ((w_pre || w_post || gate_parts) && (!ws || !q8t_aligned(ws, 16))) return Q8T_ERR_WORKSPACE;
    int sums = w_pre ? 1 : 0, post_at = -1, gate_at = -1;
    if (w_post) post_at = sums++;
    if (gate_parts) gate_at = sums++;
    const NormBack a = {dy, dres_out, res_out, h, gate, stats, w_post, w_pre, dres, dh, dgate, (float *)ws, sums, post_at, gate_at, T, D,
                        group_rows, k.rows, k.per_group, res_scale, branch_scale, d, seed, step};
    if (type == Q8T_F32) Q8T_BY_SHAPE(run_bwd, float, D, a, k.count, d.cut != 0, st);
    else Q8T_BY_SHAPE(run_bwd, q8t_bf16, D, a, k.count, d.cut != 0, st);
    Q8T_LAUNCH_CHECK();
    const int64_t columns = (w_pre ? 1 : 0) + (w_post ? 1 : 0) + (gate_parts ? groups : 0);
    if (columns) {
        const dim3 grid((D + 15) / 16, (unsigned)columns);
        if (type == Q8T_F32)
            norm_bwd_columns<<<grid, 256, 0, st>>>((const float *)ws, sums, post_at, gate_at, D, k.count, k.per_group, w_pre != nullptr, dw_pre,
                                                   dw_post, (float *)dgate);
        else
            norm_bwd_columns<<<grid, 256, 0, st>>>((const float *)ws, sums, post_at, gate_at, D, k.count, k.per_group, w_pre != nullptr, dw_pre,
                                                   dw_post, (q8t_bf16 *)dgate);
        Q8T_LAUNCH_CHECK();
    }
    return Q8T_OK;
}

}  // extern "C"
