// attn_forward_d.hip -- the attention kernels of one padded head_dim
// (KVX_ATTN_DP = 64, 128 or 256), both dtypes.
#include "attn_forward_kernels.h"

namespace kvx {

template <typename T, int DP>
hipError_t run_forward(const AttnArgs& a, const ForwardPlan& p, hipStream_t st) {
  return run_attention<T, DP>(a, p, st);
}

template hipError_t run_forward<float, KVX_ATTN_DP>(const AttnArgs&, const ForwardPlan&, hipStream_t);
template hipError_t run_forward<bf16_t, KVX_ATTN_DP>(const AttnArgs&, const ForwardPlan&, hipStream_t);

}  // namespace kvx
