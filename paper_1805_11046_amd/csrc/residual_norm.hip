// Norms behind and in front of a block with its gate, residual scales and drop-out: entry points, and the sums over rows of the backward
// pass (kernels over rows: residual_norm.h).
#include "residual_norm.h"

namespace {

// Column sums of the chunks' partial sums, in one order whatever the launch: 32 columns x 32 threads of four columns, each over every
// 32nd chunk: 5.7 us for three sums of 5120 over 250 chunks.  y = 0: dw_pre, 1: dw_post (over all chunks), from 2 on (or what is wanted of them): one group of the gate.
template <class T>
__global__ __launch_bounds__(256) void norm_bwd_columns(const float *__restrict__ part, int sums, int post_at, int gate_at, int D,
                                                        int64_t chunks, int64_t group_chunks, bool pre, float *dw_pre, float *dw_post,
                                                        T *dgate)
{
    __shared__ float fold[32][33];
    const int tx = threadIdx.x & 7, ty = threadIdx.x / 8, width = norm_part_width(D);
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
    const float *p = part + (first * sums + at) * width + blockIdx.x * 32 + tx * 4;
    const int64_t step = (int64_t)sums * width;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
    for (int64_t k = ty; k < count; k += 32) {
        const float4 w = *reinterpret_cast<const float4 *>(p + k * step);
        v[0] += w.x, v[1] += w.y, v[2] += w.z, v[3] += w.w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) fold[ty][tx * 4 + i] = v[i];
    __syncthreads();
    const int col = threadIdx.x & 31, c = blockIdx.x * 32 + col, eighth = threadIdx.x / 32;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) s += fold[eighth + 8 * i][col];
    __syncthreads();
    fold[eighth][col] = s;
    __syncthreads();
    if (eighth || c >= D) return;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += fold[i][col];
    if (z >= weights) dgate[(z - weights) * D + c] = (T)s;
    else (at == post_at ? dw_post : dw_pre)[c] = s;
}

template <class T>
__global__ __launch_bounds__(256) void clear(T *p, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = (T)0.0f;
}

// Chunks of rows of the backward pass, a workgroup each: as many as the chip holds at 16 wavefronts a compute unit (128 registers), up to 2048,
// because every chunk costs D (2 or 3 times) partial sums, written and read again; for the same reason chunks of fewer than four rows only
// where there would be fewer than one a compute unit.  bf16, us, with 256, 512, 1024, 2048 chunks: 1000 x 16384 94, 116, 167, 168;
// 6000 x 5120 89, 94, 107, 132; 8192 x 4096 93, 83, 91, 108; 8192 x 2048 81, 51, 48, 59; 2048 x 1024 24, 19, 20, 24; 32768 x 1024 249, 142, 92, 82.
// Groups shorter than a chunk are taken whole (their gate's gradient is final there), longer ones are cut.
struct Chunks {
    int64_t rows, per_group, count;
};
Chunks chunks_of(int64_t T, int D, int64_t group_rows)
{
    const int64_t fit = 16 / (norm_threads(D) / 64), most = 256 * (fit < 1 ? 1 : (fit > 8 ? 8 : fit));
    const int64_t few = (T + 255) / 256;
    int64_t rows = (T + most - 1) / most;
    if (rows < 4) rows = few < 4 ? few : 4;
    if (group_rows <= rows) {
        rows = (rows + group_rows - 1) / group_rows * group_rows;
        return {rows, 0, (T + rows - 1) / rows};
    }
    const int64_t per = (group_rows + rows - 1) / rows;   // at least two; there are fewer than `most` groups to cut
    return {(group_rows + per - 1) / per, per, per * (T / group_rows)};
}

int check(int type, int64_t T, int D, int64_t groups, double p, Q8tDrop *d)
{
    if (T < 0 || D < 1 || D > kNormMaxD || groups < 0 || (groups > 0 && T % groups)) return Q8T_ERR_SHAPE;
    if (T > ((int64_t)1 << 34) / D || T >= (int64_t)1 << 22) return Q8T_ERR_SHAPE;
    if ((type != Q8T_F32 && type != Q8T_BF16) || !q8t_drop(p, d)) return Q8T_ERR_VALUE;
    return Q8T_OK;
}

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
    const Norm a = {res, h, gate, w_post, w_pre, res_out, y, stats, q, s, T, D, groups ? T / groups : 1, eps, res_scale, branch_scale, d, seed, step};
    const NormCall c = {h != nullptr, w_post != nullptr, gate != nullptr, d.cut != 0};
    (type == Q8T_F32 ? q8t_norm_fwd_f32 : q8t_norm_fwd_bf16)(a, c, (hipStream_t)stream);
    Q8T_LAUNCH_CHECK();
    return Q8T_OK;
}

size_t q8t_residual_norm_bwd_workspace_size(int64_t T, int D, int64_t groups)
{
    if (T <= 0 || D < 1 || D > kNormMaxD || groups < 0 || (groups > 0 && T % groups) || T >= (int64_t)1 << 22) return 0;
    return (size_t)chunks_of(T, D, groups ? T / groups : 1).count * 3 * norm_part_width(D) * sizeof(float);
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
    if (!dres || (w_pre && !res_out) || ((w_pre || w_post) && !stats)) return Q8T_ERR_NULL;
    const int64_t group_rows = groups ? T / groups : 1;
    const Chunks k = chunks_of(T, D, group_rows);
    const bool gate_parts = gate && k.per_group;
    if ((w_pre || w_post || gate_parts) && (!ws || !q8t_aligned(ws, 16))) return Q8T_ERR_WORKSPACE;
    int sums = w_pre ? 1 : 0, post_at = -1, gate_at = -1;
    if (w_post) post_at = sums++;
    if (gate_parts) gate_at = sums++;
    const NormBack a = {dy, dres_out, res_out, h, gate, stats, w_post, w_pre, dres, dh, dgate, (float *)ws, sums, post_at, gate_at, T, D,
                        group_rows, k.rows, k.per_group, res_scale, branch_scale, d, seed, step};
    const NormCall c = {h != nullptr, w_post != nullptr, gate != nullptr, d.cut != 0};
    const int run = (type == Q8T_F32 ? q8t_norm_bwd_f32 : q8t_norm_bwd_bf16)(a, c, k.count, st);
    if (run) return run;
    Q8T_LAUNCH_CHECK();
    const int64_t columns = (w_pre ? 1 : 0) + (w_post ? 1 : 0) + (gate_parts ? groups : 0);
    if (columns) {
        const dim3 grid((D + 31) / 32, (unsigned)columns);
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
