// fp8 products with fp32 results: codes widened to bf16 in registers (fp8_gemm.h).
#include "fp8_gemm.h"

int q8t_fp8_product_f32(const Fp8Product &p, int fa, int fb, const Fp8Plan &plan, void *ws, hipStream_t st)
{
    return by_format(fa, fb, [&](auto a, auto b) {
        constexpr int A = decltype(a)::value, B = decltype(b)::value;
        switch (plan.form) {
        case FP8_DIRECT_16: return run_direct<A, B, float, 1, 1>(p, st);
        case FP8_DIRECT_32: return run_direct<A, B, float, 2, 1>(p, st);
        case FP8_DIRECT_64: return run_direct<A, B, float, 2, 2>(p, st);
        case FP8_TILE_64: {
            const int rc = run_tiles<A, B, true, float, Tile<64, 64, 32, 32, 2>>(p, plan.slices, ws, st);
            return rc || plan.slices == 1 ? rc : run_fold<float>(p, plan.slices, ws, st);
        }
        case FP8_TILE_64_128: return run_tiles<A, B, true, float, Tile<64, 128, 32, 64, 2>>(p, 1, ws, st);
        case FP8_TILE_128: return run_tiles<A, B, true, float, Tile<128, 128, 64, 64, 2>>(p, 1, ws, st);
        default: return run_tiles<A, B, true, float, Tile<256, 256, 128, 64, 2>>(p, 1, ws, st);
        }
    });
}
