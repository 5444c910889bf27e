// Forward pass of the norms round a block over fp32 tensors.
#include "residual_norm.h"

void q8t_norm_fwd_f32(const Norm &a, const NormCall &c, hipStream_t st) { run_norm_fwd<float>(a, c, st); }
