// attn_cache8.hip -- conversion of caches to 8 bits and back (kvx_attn_pack,
// kvx_attn_unpack), all layers.
#include <algorithm>

#include "attn_view.h"

namespace kvx {
namespace {

constexpr int kChunk = 128;  // slots of a workgroup's turn

// The numbers of a lane, 16 bytes of a row.
template <typename T>
struct Piece {
  static constexpr int n = 16 / sizeof(T);
  T x[n];
};

// As many codes.
template <int N>
struct Codes {
  uint32_t x[N / 4];
};

// A slot's key and value rows to codes, or back: G lanes a slot, 16 bytes of plain
// numbers each, so that a wave reads and writes whole lines; lanes past head_dim
// stay idle.  A workgroup takes kChunk slots of a head, kAhead rows a lane at a time.
template <typename T, typename C, int G, bool PACK>
__global__ void __launch_bounds__(256) convert_kernel(PackArgs a, int chunks) {
  constexpr int N = Piece<T>::n, kSlots = 256 / G, kTurns = kChunk / kSlots, kAhead = kTurns < 4 ? kTurns : 4;
  const int lane = threadIdx.x % G, sub = threadIdx.x / G;
  const bool active = lane * N < a.d;
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
#pragma unroll 1
    for (int jt = j0; jt < j1; jt += kAhead * kSlots) {
      T* plain[kAhead][2];
      char* coded[kAhead][2];
      uint32_t* pair[kAhead];
      bool there[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int j = jt + i * kSlots + sub, jc = min(j, j1 - 1);
        there[i] = j < j1;
        const int32_t pb = cache_block(a.plain, b, jc), cb = cache_block(a.coded, b, jc);
        const int64_t pat = cache_offset(a.plain, pb, jc) + l * a.plain.sl + h * a.plain.sh + lane * N;
        const int64_t cat = cache_offset(a.coded, cb, jc) + l * a.coded.sl + h * a.coded.sh + lane * N;
        plain[i][0] = reinterpret_cast<T*>(a.plain.k) + pat;
        plain[i][1] = reinterpret_cast<T*>(a.plain.v) + pat;
        coded[i][0] = a.coded.k + cat;
        coded[i][1] = a.coded.v + cat;
        pair[i] = a.scale.p + l * a.scale.sl + h * a.scale.sh + scale_offset(a.coded, a.scale, cb, jc);
      }
      if constexpr (PACK) {
        Piece<T> in[kAhead][2] = {};
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (active && there[i]) in[i][e] = *reinterpret_cast<const Piece<T>*>(plain[i][e]);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          uint32_t scales = 0;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float x[N];
            uint32_t top = 0;  // bits of the largest magnitude: an infinity's or NaN's are the largest
#pragma unroll
            for (int k = 0; k < N; ++k) {
              x[k] = load_f32<T>(&in[i][e].x[k]);
              top = max(top, __float_as_uint(x[k]) & 0x7fffffffu);
            }
#pragma unroll
            for (int k = 1; k < G; k <<= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), k)));
            const bool odd = top >= 0x7f800000u;
            if (__builtin_expect(top > 0x7f000000u, 0)) {
#pragma unroll
              for (int k = 0; k < N; ++k) x[k] = odd ? 0.f : fminf(fmaxf(x[k], -0x1p127f), 0x1p127f);
              top = 0x7f000000u;
            }
            const int ex = scale_exponent<C>(__uint_as_float(top));
            const float inv = power_of_two(-ex);
            Codes<N> out;
#pragma unroll
            for (int k = 0; k < N / 4; ++k) {
              float y[4];
#pragma unroll
              for (int z = 0; z < 4; ++z) y[z] = x[4 * k + z] * inv;
              out.x[k] = encode4<C>(y);
            }
            scales |= (odd ? 0x7fc0u : __float_as_uint(power_of_two(ex)) >> 16) << 16 * e;
            if (active && there[i]) *reinterpret_cast<Codes<N>*>(coded[i][e]) = out;
          }
          if (lane == 0 && there[i]) *pair[i] = scales;
        }
      } else {
        Codes<N> in[kAhead][2] = {};
        uint32_t scales[kAhead] = {};
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          if (!active || !there[i]) continue;
          scales[i] = *pair[i];
#pragma unroll
          for (int e = 0; e < 2; ++e) in[i][e] = *reinterpret_cast<const Codes<N>*>(coded[i][e]);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float f = e ? value_scale(scales[i]) : key_scale(scales[i]);
            Piece<T> out;
#pragma unroll
            for (int k = 0; k < N / 4; ++k) {
              float y[4];
              decode4<C>(in[i][e].x[k], f, y);
#pragma unroll
              for (int z = 0; z < 4; ++z) out.x[4 * k + z] = store_cvt<T>(y[z]);
            }
            if (active && there[i]) *reinterpret_cast<Piece<T>*>(plain[i][e]) = out;
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
  constexpr int N = Piece<T>::n;
  return a.d <= 64    ? run<T, C, 64 / N>(a, pack, n_cu, st)
         : a.d <= 128 ? run<T, C, 128 / N>(a, pack, n_cu, st)
                      : run<T, C, 256 / N>(a, pack, n_cu, st);
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
