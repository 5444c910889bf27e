// fp8 products with bf16 results: the 8-bit matrix instruction (fp8_gemm.h).
#include "fp8_gemm.h"

int q8t_fp8_product_bf16(const Fp8Product &p, int fa, int fb, const Fp8Plan &plan, void *ws, hipStream_t st)
{
    typedef Tile<64, 64, 32, 32, 4> T64;
    return by_format(fa, fb, [&](auto a, auto b) {
        constexpr int A = decltype(a)::value, B = decltype(b)::value;
        switch (plan.form) {
        case FP8_DIRECT_16: return run_direct<A, B, q8t_bf16, 1, 1>(p, st);
        case FP8_DIRECT_32: return run_direct<A, B, q8t_bf16, 2, 1>(p, st);
        case FP8_DIRECT_64: return run_direct<A, B, q8t_bf16, 2, 2>(p, st);
        case FP8_TILE_64: {
            if (plan.slices == 1) return run_tiles<A, B, false, q8t_bf16, T64>(p, 1, ws, st);
            const int rc = run_tiles<A, B, false, float, T64>(p, plan.slices, ws, st);
            return rc ? rc : run_fold<q8t_bf16>(p, plan.slices, ws, st);
        }
        case FP8_TILE_64_128: return run_tiles<A, B, false, q8t_bf16, Tile<64, 128, 32, 64, 4>>(p, 1, ws, st);
        case FP8_TILE_128_DEEP: return run_tiles<A, B, false, q8t_bf16, Tile<128, 128, 64, 64, 4>>(p, 1, ws, st);
        case FP8_TILE_128: return run_tiles<A, B, false, q8t_bf16, Tile<128, 128, 64, 64, 2>>(p, 1, ws, st);
        default: return run_tiles<A, B, false, q8t_bf16, Tile<256, 256, 128, 64, 2>>(p, 1, ws, st);
        }
    });
}
