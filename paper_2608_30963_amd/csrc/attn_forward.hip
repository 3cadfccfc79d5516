// attn_forward.hip -- attention of new tokens over the cache (kvx_attn_forward).
#include "attn.h"

namespace kvx {
namespace {

// Plain form: one wave per (row, query head), 64 slots a step -- lane i takes
// the score of slot j + i, then the lanes take head_dim columns of the values.
template <typename T>
__global__ void __launch_bounds__(64) forward_simple(AttnArgs a) {
  __shared__ float qs[256];
  __shared__ float ps[64];
  __shared__ int64_t at[64];
  const int row = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  int b = 0;
  if (a.q_start) {
    while (b + 1 < a.batch && a.q_start[b + 1] <= row) ++b;
  } else {
    b = row;
  }
  const Context c = context(a, b);
  const int p = c.n - c.m + row - c.q0;
  const int lo = first_seen(a, p), hi = row < c.q0 + c.m ? min(end_seen(c, p), c.n) : 0;
  const T* q = reinterpret_cast<const T*>(a.q) + row * a.q_sr + h * a.q_sh;
  for (int i = lane; i < a.d; i += 64) qs[i] = load_f32<T>(q + i);
  __syncthreads();
  const int64_t head = (h / a.group) * a.c.sh;
  const T* kc = reinterpret_cast<const T*>(a.c.k) + head;
  const T* vc = reinterpret_cast<const T*>(a.c.v) + head;
  float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = lo; j0 < hi; j0 += 64) {
    const int j = j0 + lane;
    float s = -INFINITY;
    if (j < hi) {
      const int64_t o = cache_offset(a.c, cache_block(a.c, b, j), j);
      at[lane] = o;
      float x = 0.f;
      for (int i = 0; i < a.d; ++i) x += qs[i] * load_f32<T>(kc + o + i);
      s = score2(a, x);
    }
    float top = s;
    for (int i = 32; i; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
    const float mn = fmaxf(m, top);
    const float alpha = m == mn ? 1.f : __builtin_amdgcn_exp2f(m - mn);
    const float e = j < hi ? __builtin_amdgcn_exp2f(s - mn) : 0.f;
    m = mn;
    float sum = e;
    for (int i = 32; i; i >>= 1) sum += __shfl_xor(sum, i);
    l = l * alpha + sum;
    ps[lane] = e;
    __syncthreads();
    const int cnt = min(64, hi - j0);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      acc[k] *= alpha;
      const int i = k * 64 + lane;
      if (i < a.d)
        for (int t = 0; t < cnt; ++t) acc[k] += ps[t] * load_f32<T>(vc + at[t] + i);
    }
    __syncthreads();
  }
  T* o = reinterpret_cast<T*>(a.out) + row * a.o_sr + h * a.o_sh;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k * 64 + lane < a.d) o[k * 64 + lane] = store_cvt<T>(lo < hi ? acc[k] / l : 0.f);
  if (a.lse && lane == 0)
    a.lse[static_cast<int64_t>(row) * a.hq + h] =
        lo < hi ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY;
}

}  // namespace

size_t forward_workspace(const kvx_attn*) { return 16; }

hipError_t launch_forward(const kvx_attn* at, const AttnArgs& a, int, void*, hipStream_t st) {
  const dim3 grid(a.rows, a.hq);
  return at->dtype == KVX_F32 ? launch_on(forward_simple<float>, grid, dim3(64), st, a)
                              : launch_on(forward_simple<bf16_t>, grid, dim3(64), st, a);
}

}  // namespace kvx
