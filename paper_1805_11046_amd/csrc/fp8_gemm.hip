// q8t_fp8_gemm: argument checks (choice of a product's form: fp8_plan.h, kernels: fp8_gemm.h).
#include "fp8_gemm.h"

extern "C" {

size_t q8t_fp8_gemm_workspace_size(int M, int N, int K)
{
    if (M <= 0 || N <= 0 || K <= 0) return 0;
    size_t most = 0;
    for (int type : {(int)Q8T_F32, (int)Q8T_BF16}) {
        const Fp8Plan p = fp8_plan_of(M, N, (K - 1) / 128 + 1, type);
        if (p.slices > 1 && (size_t)p.slices * M * N * 4 > most) most = (size_t)p.slices * M * N * 4;
    }
    return most;
}

int q8t_fp8_gemm(const uint8_t *a, const uint8_t *sa, int format_a, const uint8_t *b, const uint8_t *sb, int format_b, int M, int N, int K,
                 void *out, int type, void *ws, void *stream)
{
    // 256 rows of codes are addressed in 32 bits; a launch holds fewer than 2^32 threads
    if (M < 0 || N < 0 || K <= 0 || K > 1 << 23 || M > 1 << 22 || N > 1 << 22 || (int64_t)M * N > (int64_t)1 << 36) return Q8T_ERR_SHAPE;
    if ((type != Q8T_F32 && type != Q8T_BF16) || (format_a != Q8T_E4M3 && format_a != Q8T_E5M2) ||
        (format_b != Q8T_E4M3 && format_b != Q8T_E5M2))
        return Q8T_ERR_VALUE;
    if (M == 0 || N == 0) return Q8T_OK;
    if (!a || !sa || !b || !sb || !out) return Q8T_ERR_NULL;
    if (!q8t_aligned(a, 16) || !q8t_aligned(b, 16) || !q8t_aligned(sa, 4) || !q8t_aligned(sb, 4)) return Q8T_ERR_SHAPE;
    const Fp8Product p = {a, sa, b, sb, M, N, (K + 127) / 128, fp8_row_bytes(K), fp8_scale_bytes(K), out};
    const Fp8Plan plan = fp8_plan_of(M, N, p.nk, type);
    if (plan.slices > 1 && (!ws || !q8t_aligned(ws, 16))) return Q8T_ERR_WORKSPACE;
    return (type == Q8T_F32 ? q8t_fp8_product_f32 : q8t_fp8_product_bf16)(p, format_a, format_b, plan, ws, (hipStream_t)stream);
}

}  // extern "C"
