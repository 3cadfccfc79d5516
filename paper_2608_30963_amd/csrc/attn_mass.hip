// attn_mass.hip -- attention weight that each cached token received
// (kvx_attn_mass): which kernel a call runs.
#include "attn_mass.h"

namespace kvx {

hipError_t launch_mass(const kvx_attn* at, const AttnArgs& a, int max_new, hipStream_t st) {
  const int d = at->model.head_dim, n_cu = at->n_cu;
  const bool f32 = at->dtype == KVX_F32;
  // up to 32 query rows per context: single tokens' kernel.  Measured (us; it,
  // the chunk kernel), heads 28 / 4 x 128, 16 contexts of 4096 slots: 28 rows 20.5,
  // 29.7; 56 rows 35.4, 30.7; 112 rows 67, 35; one of 128k, 28 rows: 31, 55; one of
  // 1024, heads 12 / 2, 24 rows: 8.1, 7.0
  const bool decode = a.rows == 0 || int64_t(max_new) * at->group <= 32;
  if (d <= 64) return f32 ? run_mass<float, 64>(a, decode, n_cu, st) : run_mass<bf16_t, 64>(a, decode, n_cu, st);
  if (d <= 128) return f32 ? run_mass<float, 128>(a, decode, n_cu, st) : run_mass<bf16_t, 128>(a, decode, n_cu, st);
  return f32 ? run_mass<float, 256>(a, decode, n_cu, st) : run_mass<bf16_t, 256>(a, decode, n_cu, st);
}

}  // namespace kvx
