// attn_view.hip -- attention under a view (kvx_attn_forward_view).
#include "attn_view.h"

namespace kvx {
namespace {

constexpr float kLn2 = 0.6931471805599453f;

// A wave a (row, query head), 64 slots a turn: a lane a slot's score, then a
// lane some columns of the values' sum.
template <typename S, typename T, int PER>
__global__ void __launch_bounds__(64) rows_kernel(AttnView a) {
  const int row = blockIdx.x, head = blockIdx.y, h = head / a.group, lane = threadIdx.x;
  const int b = context_of(a, row);
  const Context c = context(a, b);
  const int i = row - c.q0;
  if (i >= c.m) return;
  const Sight st = sight(a, c, i);
  const T* q = reinterpret_cast<const T*>(a.q) + row * a.q_sr + head * a.q_sh;
  const S* kc = reinterpret_cast<const S*>(a.c.k) + h * a.c.sh;
  const S* vc = reinterpret_cast<const S*>(a.c.v) + h * a.c.sh;
  float m2 = -INFINITY, l = 0.f, o[PER];
  for (int x = 0; x < PER; ++x) o[x] = 0.f;
  const int end = st.mask ? st.end : st.hi;
  for (int j0 = 0; j0 < end; j0 += 64) {
    const uint32_t bits = seen_bits(st, j0 + lane / 32 * 32);
    const bool sees = bits >> lane % 32 & 1;
    if (!__any(sees)) continue;
    float s = -INFINITY, vf = 1.f;
    int64_t at = 0;
    if (sees) {
      const int j = j0 + lane;
      const int32_t block = cache_block(a.c, b, j);
      at = cache_offset(a.c, block, j);
      float kf = 1.f;
      if (a.scale.p) {
        const int slot = a.c.table ? j - fdiv(a.c.bs, j) * static_cast<int>(a.c.bs.d) : j;
        const uint32_t pair = a.scale.p[block * a.scale.sb + h * a.scale.sh + slot * a.scale.st];
        kf = key_scale(pair);
        vf = value_scale(pair);
      }
      float x = 0.f;
      for (int e = 0; e < a.d; ++e) x += load_f32<T>(q + e) * number<S>(kc + at + e, 1.f);
      s = score2(a, x * kf);
    }
    float top = s;
    for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
    const float m = fmaxf(m2, top);
    const float alpha = m == m2 ? 1.f : __builtin_amdgcn_exp2f(m2 - m);
    m2 = m;
    const float p = sees ? __builtin_amdgcn_exp2f(s - (m == -INFINITY ? 0.f : m)) : 0.f;
    float sum = p;
    for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x);
    l = l * alpha + sum;
    for (int x = 0; x < PER; ++x) o[x] *= alpha;
    for (int r = 0; r < 64; ++r) {
      if (!__shfl(static_cast<int>(sees), r)) continue;
      const float pr = __shfl(p, r), f = __shfl(vf, r);
      const int64_t vr = static_cast<int64_t>(
          static_cast<uint64_t>(__shfl(static_cast<uint32_t>(static_cast<uint64_t>(at) >> 32), r)) << 32 |
          __shfl(static_cast<uint32_t>(at), r));
      for (int x = 0; x < PER; ++x)
        if (x * 64 + lane < a.d) o[x] += pr * number<S>(vc + vr + x * 64 + lane, f);
    }
  }
  const bool any = sees_any(st);
  T* out = reinterpret_cast<T*>(a.out) + row * a.o_sr + head * a.o_sh;
  for (int x = 0; x < PER; ++x)
    if (x * 64 + lane < a.d) out[x * 64 + lane] = store_cvt<T>(any ? o[x] / l : 0.f);
  if (a.lse && lane == 0)
    a.lse[static_cast<int64_t>(row) * a.hq + head] = any ? (m2 + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

}  // namespace

hipError_t launch_view(const kvx_attn* at, const AttnView& a, int code, int, void*, hipStream_t st) {
  const dim3 grid(a.rows, a.hq), block(64);
  return code == KVX_CODE_I8     ? launch_on(rows_kernel<code_i8, bf16_t, 4>, grid, block, st, a)
         : code == KVX_CODE_E4M3 ? launch_on(rows_kernel<code_e4m3, bf16_t, 4>, grid, block, st, a)
         : at->dtype == KVX_F32  ? launch_on(rows_kernel<float, float, 4>, grid, block, st, a)
                                 : launch_on(rows_kernel<bf16_t, bf16_t, 4>, grid, block, st, a);
}

}  // namespace kvx
