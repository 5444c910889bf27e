// Backward pass of the norms round a block over bf16 tensors.
#include "residual_norm.h"

int q8t_norm_bwd_bf16(const NormBack &a, const NormCall &c, int64_t chunks, hipStream_t st) { return run_norm_bwd<q8t_bf16>(a, c, chunks, st); }
