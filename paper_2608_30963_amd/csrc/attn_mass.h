// attn_mass.h -- the attention-weight kernels' launcher, one translation unit
// per head_dim (attn_mass_d.hip).
#pragma once

#include <algorithm>

#include "attn.h"

namespace kvx {

template <typename T, int DP>
hipError_t run_mass(const AttnArgs& a, bool decode, int n_cu, hipStream_t st);

}  // namespace kvx
