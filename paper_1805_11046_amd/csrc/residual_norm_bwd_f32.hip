// Backward pass of the norms round a block over fp32 tensors.
#include "residual_norm.h"

int q8t_norm_bwd_f32(const NormBack &a, const NormCall &c, int64_t chunks, hipStream_t st) { return run_norm_bwd<float>(a, c, chunks, st); }
