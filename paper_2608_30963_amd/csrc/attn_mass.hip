// attn_mass.hip -- attention weight that each cached token received
// (kvx_attn_mass).
#include "attn.h"

namespace kvx {
namespace {

// Plain form: one thread per (context, KV head, slot).
template <typename T>
__global__ void __launch_bounds__(64) mass_simple(AttnArgs a) {
  const int j = blockIdx.x * 64 + threadIdx.x, h = blockIdx.y, b = blockIdx.z;
  if (j >= a.mass_capacity) return;
  const int64_t at = (static_cast<int64_t>(b) * a.hkv + h) * a.mass_capacity + j;
  float sum = 0.f;
  const Context c = context(a, b);
  if (j < c.n) {
    const T* k = nullptr;
    for (int i = 0; i < c.m; ++i) {
      const int p = c.n - c.m + i;
      if (j < first_seen(a, p) || j >= end_seen(c, p)) continue;
      if (!k)
        k = reinterpret_cast<const T*>(a.c.k) + cache_offset(a.c, cache_block(a.c, b, j), j) +
            h * a.c.sh;
      const int64_t row = c.q0 + i;
      for (int g = 0; g < a.group; ++g) {
        const int qh = h * a.group + g;
        const T* q = reinterpret_cast<const T*>(a.q) + row * a.q_sr + qh * a.q_sh;
        float x = 0.f;
        for (int e = 0; e < a.d; ++e) x += load_f32<T>(q + e) * load_f32<T>(k + e);
        sum += __builtin_amdgcn_exp2f(score2(a, x) - a.lse[row * a.hq + qh] * 1.4426950408889634f);
      }
    }
  }
  a.mass[at] = (a.mass_in ? a.mass_in[at] : 0.f) + sum;
}

}  // namespace

hipError_t launch_mass(const kvx_attn* at, const AttnArgs& a, int, hipStream_t st) {
  const dim3 grid((a.mass_capacity + 63) / 64, a.hkv, a.batch);
  return at->dtype == KVX_F32 ? launch_on(mass_simple<float>, grid, dim3(64), st, a)
                              : launch_on(mass_simple<bf16_t>, grid, dim3(64), st, a);
}

}  // namespace kvx
