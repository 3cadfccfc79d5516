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

// Slots' key and value rows to codes, or back: G lanes a slot, 16 bytes of plain
// numbers each, so that a wave reads and writes whole lines; lanes past head_dim
// stay idle.  A workgroup's turn is kChunk slots of a head, a wave's 16 of them,
// whose rows are all asked for before the first is worked on.  Bound by memory:
// 28 layers of 4k slots, 2 heads x 128, bf16 to int8: 176 MB in 41.5 us, 4.2 TB/s; 26
// layers, 4 contexts of up to 2k slots, 4 heads x 256, e4m3 to bf16: 887 MB in 201 us,
// 4.4 TB/s (by 8 bytes of codes a lane and one row at a time: 289).
// Where 16 slots from a multiple of 16 on lie in one block of both caches, a
// wave's rows have one base; else every lane finds its own.
template <typename T, typename C, int G, bool PACK>
__global__ void __launch_bounds__(256) convert_kernel(PackArgs a, int chunks) {
  constexpr int N = Piece<T>::n, kRows = 64 / G;              // slots of a wave's instruction
  constexpr int kAhead = 16 / kRows < 4 ? 16 / kRows : 4;     // of them at a time
  const int lane = threadIdx.x % 64, piece = lane % G, sub = lane / G;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const bool active = piece * N < a.d, based = a.plain.run >= 16 && a.coded.run >= 16;
  const int64_t sets = int64_t(a.layers) * a.batch * a.heads;
  for (int64_t id = blockIdx.x; id < sets * chunks; id += gridDim.x) {
    const int64_t set = id / chunks;
    const int j0 = static_cast<int>(id - set * chunks) * kChunk;
    const int h = static_cast<int>(set % a.heads);
    const int64_t lb = set / a.heads;
    const int b = static_cast<int>(lb % a.batch);
    const int64_t l = lb / a.batch;
    const int n = min(min(max(a.tokens[b], 0), a.plain.capacity), a.coded.capacity);
    const int64_t plain0 = l * a.plain.sl + h * a.plain.sh, coded0 = l * a.coded.sl + h * a.coded.sh;
    const int64_t pair0 = l * a.scale.sl + h * a.scale.sh;
#pragma unroll 1
    for (int jw = j0 + 16 * w; jw < min(n, j0 + kChunk); jw += 64) {
      const int rows = min(16, n - jw);
      int64_t pb = plain0, cb = coded0, sb = pair0;  // of slot jw
      if (based) {
        const int32_t p = cache_block(a.plain, b, jw), c = cache_block(a.coded, b, jw);
        pb += cache_offset(a.plain, p, jw);
        cb += cache_offset(a.coded, c, jw);
        sb += scale_offset(a.coded, a.scale, c, jw);
      }
#pragma unroll 1
      for (int r0 = 0; r0 < rows; r0 += kAhead * kRows) {
        int64_t pat[kAhead], cat[kAhead], sat[kAhead];
        bool there[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int r = r0 + i * kRows + sub;
          there[i] = r < rows;
          if (based) {
            pat[i] = pb + static_cast<int64_t>(r * static_cast<uint64_t>(a.plain.st));
            cat[i] = cb + static_cast<int64_t>(r * static_cast<uint64_t>(a.coded.st));
            sat[i] = sb + r * a.scale.st;
          } else {
            const int j = jw + min(r, rows - 1);
            const int32_t p = cache_block(a.plain, b, j), c = cache_block(a.coded, b, j);
            pat[i] = plain0 + cache_offset(a.plain, p, j);
            cat[i] = coded0 + cache_offset(a.coded, c, j);
            sat[i] = pair0 + scale_offset(a.coded, a.scale, c, j);
          }
          pat[i] += piece * N;
          cat[i] += piece * N;
        }
        T* const pk[2] = {reinterpret_cast<T*>(a.plain.k), reinterpret_cast<T*>(a.plain.v)};
        char* const ck[2] = {a.coded.k, a.coded.v};
        if constexpr (PACK) {
          Piece<T> in[kAhead][2] = {};
#pragma unroll
          for (int i = 0; i < kAhead; ++i)
            if (active && there[i])
#pragma unroll
              for (int e = 0; e < 2; ++e) in[i][e] = *reinterpret_cast<const Piece<T>*>(pk[e] + pat[i]);
#pragma unroll
          for (int i = 0; i < kAhead; ++i) {
            uint32_t scales = 0;
            Codes<N> out[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float x[N];
#pragma unroll
              for (int k = 0; k < N; ++k) x[k] = load_f32<T>(&in[i][e].x[k]);
              scales |= encode_row<C, G>(x, out[e].x) << 16 * e;
            }
            if (active && there[i]) {
#pragma unroll
              for (int e = 0; e < 2; ++e) *reinterpret_cast<Codes<N>*>(ck[e] + cat[i]) = out[e];
              if (piece == 0) a.scale.p[sat[i]] = scales;
            }
          }
        } else {
          Codes<N> in[kAhead][2] = {};
          uint32_t scales[kAhead] = {};
#pragma unroll
          for (int i = 0; i < kAhead; ++i)
            if (active && there[i]) {
              scales[i] = a.scale.p[sat[i]];
#pragma unroll
              for (int e = 0; e < 2; ++e) in[i][e] = *reinterpret_cast<const Codes<N>*>(ck[e] + cat[i]);
            }
#pragma unroll
          for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float f = e ? value_scale(scales[i]) : key_scale(scales[i]);
              Piece<T> out;
              if constexpr (N == 8) {
                out = __builtin_bit_cast(Piece<T>, code_numbers<C>(in[i][e].x[0], in[i][e].x[1], f));
              } else {
                float y[4];
                decode4<C>(in[i][e].x[0], f, y);
                out = __builtin_bit_cast(Piece<T>, y);
              }
              if (active && there[i]) *reinterpret_cast<Piece<T>*>(pk[e] + pat[i]) = out;
            }
        }
      }
    }
  }
}

template <typename T, typename C, int G>
hipError_t run(const PackArgs& a, bool pack, int n_cu, hipStream_t st) {
  const int chunks = (std::min(a.plain.capacity, a.coded.capacity) + kChunk - 1) / kChunk;
  const int64_t items = int64_t(a.layers) * a.batch * a.heads * chunks;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(items, 128 * int64_t(n_cu))));
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
