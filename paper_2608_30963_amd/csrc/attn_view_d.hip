// attn_view_d.hip -- the attention kernels under a view of one padded head_dim
// (KVX_ATTN_DP = 64, 128 or 256), over caches of the model's dtype, or with
// KVX_ATTN_CODED of 8 bits.
#include "attn_forward_kernels.h"

namespace kvx {

template <typename S, int DP>
hipError_t run_view(const AttnView& a, const ForwardPlan& p, hipStream_t st) {
  return run_attention<S, DP>(a, p, st);
}

#if KVX_ATTN_CODED
template hipError_t run_view<code_i8, KVX_ATTN_DP>(const AttnView&, const ForwardPlan&, hipStream_t);
template hipError_t run_view<code_e4m3, KVX_ATTN_DP>(const AttnView&, const ForwardPlan&, hipStream_t);
#else
template hipError_t run_view<float, KVX_ATTN_DP>(const AttnView&, const ForwardPlan&, hipStream_t);
template hipError_t run_view<bf16_t, KVX_ATTN_DP>(const AttnView&, const ForwardPlan&, hipStream_t);
#endif

}  // namespace kvx
