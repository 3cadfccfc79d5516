// attn_cache8.hip -- conversion of caches to 8 bits and back (kvx_attn_pack,
// kvx_attn_unpack), all layers.
#include <algorithm>

#include "attn_view.h"

namespace kvx {
namespace {

constexpr int kChunk = 128;  // slots of a workgroup's turn

// 16 numbers of a row.
template <typename T>
struct Numbers {
  static constexpr int kPieces = sizeof(T);  // of 16 bytes
  uint4 x[kPieces];
};

template <typename T>
__device__ __forceinline__ void widen(const Numbers<T>& in, float (&x)[16]) {
  const T* p = reinterpret_cast<const T*>(in.x);
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = load_f32<T>(p + i);
}

// A slot's key and value rows to codes, or back.  G lanes a slot, 16 numbers of
// each row a lane; lanes past head_dim stay idle.
template <typename T, typename C, int G, bool PACK>
__global__ void __launch_bounds__(256) convert_kernel(PackArgs a, int chunks) {
  const int lane = threadIdx.x % G, sub = threadIdx.x / G;
  const bool active = lane * 16 < a.d;
  const int64_t sets = int64_t(a.layers) * a.batch * a.heads;
  for (int64_t id = blockIdx.x; id < sets * chunks; id += gridDim.x) {
    const int64_t set = id / chunks;
    const int j0 = static_cast<int>(id - set * chunks) * kChunk;
    const int h = static_cast<int>(set % a.heads);
    const int64_t lb = set / a.heads;
    const int b = static_cast<int>(lb % a.batch);
    const int64_t l = lb / a.batch;
    const int n = min(min(max(a.tokens[b], 0), a.plain.capacity), a.coded.capacity);
    const int j1 = min(n, j0 + kChunk);
    for (int j = j0 + sub; j - sub < j1; j += 256 / G) {
      const bool there = j < j1;
      const int jc = min(j, j1 - 1);
      const int32_t pb = cache_block(a.plain, b, jc), cb = cache_block(a.coded, b, jc);
      const int64_t pat = cache_offset(a.plain, pb, jc) + l * a.plain.sl + h * a.plain.sh;
      const int64_t cat = cache_offset(a.coded, cb, jc) + l * a.coded.sl + h * a.coded.sh;
      const int slot = a.coded.table ? jc - fdiv(a.coded.bs, jc) * static_cast<int>(a.coded.bs.d) : jc;
      uint32_t* pair = a.scale.p + l * a.scale.sl + cb * a.scale.sb + h * a.scale.sh + slot * a.scale.st;
      if constexpr (PACK) {
        uint32_t scales = 0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          Numbers<T> in{};
          if (active) in = *reinterpret_cast<const Numbers<T>*>((e ? a.plain.v : a.plain.k) + (pat + lane * 16) * int64_t(sizeof(T)));
          float x[16];
          widen(in, x);
          float top = 0.f;
          bool odd = false;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            odd |= (__float_as_uint(x[i]) & 0x7f800000u) == 0x7f800000u;
            x[i] = fminf(fmaxf(x[i], -0x1p127f), 0x1p127f);
            top = fmaxf(top, fabsf(x[i]));
          }
          int odds = odd;
#pragma unroll
          for (int i = 1; i < G; i <<= 1) {
            top = fmaxf(top, __shfl_xor(top, i));
            odds |= __shfl_xor(odds, i);
          }
          const int ex = scale_exponent<C>(top);
          const float inv = odds ? 0.f : power_of_two(-ex);
          uint32_t u[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = odds ? 0.f : x[4 * i + k] * inv;
            u[i] = encode4<C>(y);
          }
          scales |= (odds ? 0x7fc0u : __float_as_uint(power_of_two(ex)) >> 16) << 16 * e;
          if (active && there)
            *reinterpret_cast<uint4*>((e ? a.coded.v : a.coded.k) + cat + lane * 16) = uint4{u[0], u[1], u[2], u[3]};
        }
        if (lane == 0 && there) *pair = scales;
      } else {
        if (!there || !active) continue;
        const uint32_t scales = *pair;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint4 in = *reinterpret_cast<const uint4*>((e ? a.coded.v : a.coded.k) + cat + lane * 16);
          const uint32_t u[4] = {in.x, in.y, in.z, in.w};
          const float f = e ? value_scale(scales) : key_scale(scales);
          Numbers<T> out;
          T* o = reinterpret_cast<T*>(out.x);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float y[4];
            decode4<C>(u[i], f, y);
#pragma unroll
            for (int k = 0; k < 4; ++k) o[4 * i + k] = store_cvt<T>(y[k]);
          }
          *reinterpret_cast<Numbers<T>*>((e ? a.plain.v : a.plain.k) + (pat + lane * 16) * int64_t(sizeof(T))) = out;
        }
      }
    }
  }
}

template <typename T, typename C, int G>
hipError_t run(const PackArgs& a, bool pack, int n_cu, hipStream_t st) {
  const int chunks = (std::min(a.plain.capacity, a.coded.capacity) + kChunk - 1) / kChunk;
  const int64_t items = int64_t(a.layers) * a.batch * a.heads * chunks;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(items, 8 * int64_t(n_cu))));
  return pack ? launch_on(convert_kernel<T, C, G, true>, grid, dim3(256), st, a, chunks)
              : launch_on(convert_kernel<T, C, G, false>, grid, dim3(256), st, a, chunks);
}

template <typename T, typename C>
hipError_t by_width(const PackArgs& a, bool pack, int n_cu, hipStream_t st) {
  return a.d <= 64    ? run<T, C, 4>(a, pack, n_cu, st)
         : a.d <= 128 ? run<T, C, 8>(a, pack, n_cu, st)
                      : run<T, C, 16>(a, pack, n_cu, st);
}

}  // namespace

hipError_t launch_pack(const kvx_attn* at, const PackArgs& a, int code, bool pack, hipStream_t st) {
  if (at->dtype == KVX_F32)
    return code == KVX_CODE_I8 ? by_width<float, code_i8>(a, pack, at->n_cu, st)
                               : by_width<float, code_e4m3>(a, pack, at->n_cu, st);
  return code == KVX_CODE_I8 ? by_width<bf16_t, code_i8>(a, pack, at->n_cu, st)
                             : by_width<bf16_t, code_e4m3>(a, pack, at->n_cu, st);
}

}  // namespace kvx
