// attn_view.h -- what a row sees under a view (kvx_serve.h), and caches of 8
// bits: codes, their scales and their numbers.
#pragma once

#include "attn.h"
#include "kvx_serve.h"

namespace kvx {

// Numbers of 8 bits, as the types of a cache.
struct code_i8 {
  uint8_t x;
};
struct code_e4m3 {
  uint8_t x;
};

// Where scales lie: those of slot j of context b and head h are pair block * sb
// + h * sh + (j % block_size) * st, the block and block_size the codes'.
struct ScaleArgs {
  uint32_t* p;  // low half: the key's bf16, high half: the value's
  int64_t sl, sb, sh, st;
};

// One layer's forward under a view.
struct AttnView : AttnArgs {
  int32_t sink;
  const uint32_t* tree;  // NULL: none
  int32_t words;
  const int32_t* depth;  // NULL: rows in order
  ScaleArgs scale;       // caches of 8 bits
};

// The slots that one row sees: [lo, hi), [0, sink) below hi, and the set bits of
// mask, bit k standing for slot p0 + k, below end.
struct Sight {
  int lo, hi, sink;
  int p0, end, words;
  const uint32_t* mask;  // NULL: none
};

__device__ __forceinline__ Sight sight(const AttnView& a, const Context& c, int i) {
  Sight s;
  const int p = c.p0 + i;  // slot
  s.p0 = c.p0;
  s.end = c.n;
  s.words = a.words;
  s.mask = nullptr;
  if (a.tree) {
    const int64_t row = static_cast<int64_t>(c.q0) + i;
    const int d = a.depth ? min(max(a.depth[row], 0), max(c.m - 1, 0)) : i;
    s.lo = first_seen(a, c.p0 + d);
    s.hi = p < 0 ? 0 : min(max(c.p0, 0), c.n);
    if (p >= 0) s.mask = a.tree + row * a.words;
  } else {
    s.lo = first_seen(a, p);
    s.hi = end_seen(c, p);
  }
  s.lo = min(s.lo, s.hi);
  s.sink = min(a.sink, s.hi);
  return s;
}

__device__ __forceinline__ uint32_t low_bits(int n) {
  return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
}

// Pair of slot j in block `block`, of head 0.
__device__ __forceinline__ int64_t scale_offset(const CacheArgs& c, const ScaleArgs& s, int32_t block, int j) {
  const int slot = c.table ? j - fdiv(c.bs, j) * static_cast<int>(c.bs.d) : j;
  return block * s.sb + slot * s.st;
}

// Which of the slots j0 .. j0 + 31 the row sees, slot j0 + i in bit i.
__device__ __forceinline__ uint32_t seen_bits(const Sight& s, int j0) {
  uint32_t bits = low_bits(s.hi - j0) & (~low_bits(s.lo - j0) | low_bits(s.sink - j0));
  if (s.mask && j0 + 32 > s.p0 && j0 < s.end) {
    const int o = j0 - s.p0, w = o >> 5;
    const uint64_t lo = w >= 0 && w < s.words ? s.mask[w] : 0u;
    const uint64_t hi = w + 1 >= 0 && w + 1 < s.words ? s.mask[w + 1] : 0u;
    bits |= static_cast<uint32_t>((hi << 32 | lo) >> (o & 31)) & low_bits(s.end - j0);
  }
  return bits;
}

// Whether the row sees anything.
__device__ __forceinline__ bool sees_any(const Sight& s) {
  if (s.lo < s.hi || s.sink > 0) return true;
  if (!s.mask) return false;
  uint32_t any = 0;
  const int first = max(0, -s.p0);  // nodes of negative slots are not there
  for (int w = 0; w < s.words; ++w)
    any |= s.mask[w] & ~low_bits(first - 32 * w) & low_bits(s.end - s.p0 - 32 * w);
  return any != 0;
}

// ---------------------------------------------------------------------------
// Codes
// ---------------------------------------------------------------------------

// A row's scale 2^e by its largest magnitude, taken from that number's bits:
// top = f 2^k, f in [1/2, 1), and the largest code is M = g 2^r, g of f's range,
// so that top <= M 2^e from e = k - r on, or one more where f > g.
template <typename C>
__device__ __forceinline__ int scale_exponent(float top) {
  constexpr bool kI8 = std::is_same<C, code_i8>::value;
  const uint32_t b = __float_as_uint(top);
  const uint32_t past = (b & 0x7fffffu) > (kI8 ? 0x7e0000u : 0x600000u) ? 1 : 0;
  return max(static_cast<int>((b >> 23) + past) - 126 - (kI8 ? 7 : 9), -100);
}

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// Codes of four numbers that are already divided by their scale.  Integers: beside
// 1.5 * 2^23 a number is rounded to one, whose low byte is the sum's.
template <typename C>
__device__ __forceinline__ uint32_t encode4(const float (&x)[4]) {
  if constexpr (std::is_same<C, code_i8>::value) {
    uint32_t y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = __float_as_uint(x[i] + 12582912.f);
    const uint32_t lo = __builtin_amdgcn_perm(y[1], y[0], 0x0c0c0400), hi = __builtin_amdgcn_perm(y[3], y[2], 0x04000c0c);
    return lo | hi;
  } else {
    int u = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], u, true));
  }
}

// The numbers of four codes, times a scale.
template <typename C>
__device__ __forceinline__ void decode4(uint32_t u, float scale, float (&x)[4]) {
  if constexpr (std::is_same<C, code_i8>::value) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = static_cast<float>(static_cast<signed char>(u >> 8 * i)) * scale;
  } else {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(u, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(u, true);
    x[0] = a[0] * scale;
    x[1] = a[1] * scale;
    x[2] = b[0] * scale;
    x[3] = b[1] * scale;
  }
}

// Eight codes as bf16, which holds them exactly.
template <typename C>
__device__ __forceinline__ bf16x8 code_numbers(uint32_t a, uint32_t b, float scale = 1.f) {
  union {
    uint32_t u[4];
    bf16x8 x;
  } r;
  const uint32_t w[2] = {a, b};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (std::is_same<C, code_e4m3>::value) {
      // the instruction takes the scale's exponent, and gives NaN for a NaN
      r.u[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false));
      r.u[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true));
    } else {
      float f[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = static_cast<float>(static_cast<signed char>(w[i] >> 8 * e)) * scale;
      // their upper halves: the lower ones are zero
      r.u[2 * i] = __builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302);
      r.u[2 * i + 1] = __builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302);
    }
  }
  return r.x;
}

// One number of a row.
template <typename S>
__device__ __forceinline__ float number(const S* p, float scale) {
  if constexpr (sizeof(S) == 1) {
    float x[4];
    decode4<S>(p->x, scale, x);
    return x[0];
  } else {
    return load_f32<S>(p);
  }
}

// The largest x of G lanes (a power of two of them side by side), in all of them.
template <int G>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
  auto other = [&](auto ctrl) {
    return static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  // lanes 1 and 2 on within four, mirrored within 8 and 16, rows and halves swapped
  if constexpr (G > 1) x = max(x, other(std::integral_constant<int, 0xb1>{}));
  if constexpr (G > 2) x = max(x, other(std::integral_constant<int, 0x4e>{}));
  if constexpr (G > 4) x = max(x, other(std::integral_constant<int, 0x141>{}));
  if constexpr (G > 8) x = max(x, other(std::integral_constant<int, 0x140>{}));
  if constexpr (G > 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max(r[0], r[1]);
  }
  if constexpr (G > 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    x = max(r[0], r[1]);
  }
  return x;
}

// Codes of a lane's share of a row: G lanes' numbers x (of which lanes past the
// row's end have zeros).  Returns the bf16 of the row's scale.  x is used up.
template <typename C, int G, int N>
__device__ __forceinline__ uint32_t encode_row(float (&x)[N], uint32_t (&u)[N / 4]) {
  uint32_t top = 0;  // bits of the largest magnitude: an infinity's or NaN's are the largest
#pragma unroll
  for (int k = 0; k < N; ++k) top = max(top, __float_as_uint(x[k]) & 0x7fffffffu);
  top = group_max<G>(top);
  const bool odd = top >= 0x7f800000u;
  if (__builtin_expect(top > 0x7f000000u, 0)) {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = odd ? 0.f : fminf(fmaxf(x[k], -0x1p127f), 0x1p127f);
    top = 0x7f000000u;
  }
  const int ex = scale_exponent<C>(__uint_as_float(top));
  const float inv = power_of_two(-ex);
#pragma unroll
  for (int k = 0; k < N / 4; ++k) {
    float y[4];
#pragma unroll
    for (int z = 0; z < 4; ++z) y[z] = x[4 * k + z] * inv;
    u[k] = encode4<C>(y);
  }
  return odd ? 0x7fc0u : __float_as_uint(power_of_two(ex)) >> 16;
}

__device__ __forceinline__ float key_scale(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float value_scale(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }

struct PackArgs {
  CacheArgs plain, coded;  // all layers
  ScaleArgs scale;
  const int32_t* tokens;
  int32_t layers, batch, heads, d;
};

struct TreeArgs {
  int32_t batch, rows, axes;
  const int32_t* q_start;
  const int32_t* tokens;
  const int32_t* parent;
  int32_t window, sink;
  const int32_t* shift;
  int32_t words;
  uint32_t* mask;
  int32_t* depth;
  int32_t* pos;
};

struct AcceptArgs {
  CacheArgs c;  // all layers
  ScaleArgs scale;  // p NULL: none
  const int32_t* q_start;
  const int32_t* tokens;
  const int32_t* path;
  int32_t max_path;
  const int32_t* count;
  int32_t* tokens_out;
  int32_t layers, batch, heads, row_bytes, es;
};

// Launchers; each returns the launch's own status.
hipError_t launch_pack(const kvx_attn* at, const PackArgs& a, int code, bool pack, hipStream_t st);
hipError_t launch_tree(const TreeArgs& a, hipStream_t st);
hipError_t launch_accept(const kvx_attn* at, const AcceptArgs& a, hipStream_t st);
// code: kvx_code of the cache, -1: the model's dtype
hipError_t launch_view(const kvx_attn* at, const AttnView& a, int code, int max_new, void* workspace,
                       hipStream_t st);

}  // namespace kvx
