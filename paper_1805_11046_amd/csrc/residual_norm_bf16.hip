// Forward pass of the norms round a block over bf16 tensors.
#include "residual_norm.h"

void q8t_norm_fwd_bf16(const Norm &a, const NormCall &c, hipStream_t st) { run_norm_fwd<q8t_bf16>(a, c, st); }
