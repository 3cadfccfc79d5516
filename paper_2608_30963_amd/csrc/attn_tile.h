// attn_tile.h -- what the attention kernels do with a tile of 32 slots and 32
// query rows: its copy into LDS, the scores, the softmax step and the product
// with the values.
//
// Scores are taken transposed, S^T = K Q^T (32 x 32 matrix instructions): lane
// (n, h) = (lane % 32, lane / 32) holds query n's scores of slots 8 (v / 4) +
// 4 h + v % 4 in register v.  A query's maximum and sum are then within two
// lanes, and the weights already lie as the second product O^T = V^T P^T wants
// its right operand, if its contraction takes the slots in that order too: the
// values' operand is read in it.  O^T holds query n in lane n, so rescaling is
// by the lane's own factor.
#pragma once

#include "attn.h"

namespace kvx {

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// s_waitcnt immediate: at most n vector-memory operations outstanding.
constexpr int vm_le(int n) {
  const int m = n > 63 ? 63 : n;
  return (m & 15) | ((m >> 4) << 14) | (7 << 4) | (15 << 8);
}

// Workgroup barrier for LDS that leaves vector-memory operations in flight.
__device__ __forceinline__ void tile_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Both halves' values of x (the lane's own and lane ^ 32's).
__device__ __forceinline__ void both_halves(float x, float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}
__device__ __forceinline__ float half_max(float x) {
  float a, b;
  both_halves(x, a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float half_sum(float x) {
  float a, b;
  both_halves(x, a, b);
  return a + b;
}

__device__ __forceinline__ bool finite(float x) {
  return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u;
}

// Rows of head_dim DP (padded with zeros past a.d) in LDS: 16-byte chunk c of
// row r lies at chunk c ^ (r % 16) of its row (r % 8 where a row has 8
// chunks), which spreads the rows that one read instruction touches over the
// banks.
template <typename T, int DP>
struct Tile {
  static constexpr int kChunks = DP * sizeof(T) / 16;
  static constexpr int kSwz = (kChunks < 16 ? kChunks : 16) - 1;
  static constexpr int kRowBytes = DP * sizeof(T);
  static constexpr int kRowsPerCopy = 64 / kChunks;  // rows of one wave's copy instruction
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int kQ = kBf16 ? DP / 16 : DP / 8;  // 16-byte query pieces of a lane

  static __device__ __forceinline__ int chunk_at(int r, int c) {
    return r * kRowBytes + ((c ^ (r & kSwz)) * 16);
  }

  // The query operand: lane (n, h) holds chunks 2 s + h of query row n.
  static __device__ __forceinline__ void load_q(uint4 (&q)[kQ], const T* row, int d) {
    const int h = (threadIdx.x % 64) / 32;
    constexpr int per = 16 / sizeof(T);
#pragma unroll
    for (int s = 0; s < kQ; ++s) {
      const int e = (2 * s + h) * per;
      q[s] = row && e < d ? *reinterpret_cast<const uint4*>(row + e) : uint4{0, 0, 0, 0};
    }
  }

  // Scores of the 32 slots whose keys start at LDS address k.
  static __device__ __forceinline__ f32x16 scores(const char* k, const uint4 (&q)[kQ]) {
    const int lane = threadIdx.x % 64, n = lane % 32, h = lane / 32;
    f32x16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
    for (int i = 0; i < kQ; ++i) {
      if constexpr (kBf16) {
        const bf16x8 a = *reinterpret_cast<const bf16x8*>(k + chunk_at(n, 2 * i + h));
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, q[i]), s, 0, 0, 0);
      } else {
        const f32x4 a = *reinterpret_cast<const f32x4*>(k + chunk_at(n, 2 * i + h));
        const f32x4 b = __builtin_bit_cast(f32x4, q[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], s, 0, 0, 0);
      }
    }
    return s;
  }

  // The values' operand of 16 slots (k-step ks of the tile) and 32 columns
  // (block db): lane (m, h) holds column 32 db + m of slots 16 ks + 4 h + 0..3
  // and 16 ks + 8 + 4 h + 0..3.  The transposing read hands lane i of 16 the
  // i-th column of the 4 rows whose 16 columns the lanes' addresses name.
  static __device__ __forceinline__ bf16x8 value_frag(const char* v, int ks, int db) {
    const int lane = threadIdx.x % 64, i = lane % 16, h = lane / 32;
    const int c = 4 * db + 2 * (lane / 16 % 2) + i % 4 / 2;
    s16x4 r[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = 16 * ks + 8 * e + 4 * h + i / 4;
      r[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_s16x4*)(v + chunk_at(row, c) + i % 2 * 8));
    }
    union {
      s16x4 s[2];
      bf16x8 b;
    } u;
    u.s[0] = r[0];
    u.s[1] = r[1];
    return u.b;
  }

  // acc += P V over the tile's 32 slots; CLEAN: values that are not finite
  // count as zero (add_odd_values has them).
  template <bool CLEAN>
  static __device__ __forceinline__ void add_values(const char* v, const f32x16& p,
                                                    f32x16 (&acc)[DP / 32]) {
    const int lane = threadIdx.x % 64;
    if constexpr (kBf16) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        // weights rounded once to bf16 for the matrix instruction; the sum
        // that divides them keeps fp32
        bf16x8 b;
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = static_cast<__bf16>(p[8 * ks + e]);
#pragma unroll
        for (int db = 0; db < DP / 32; ++db) {
          bf16x8 a = value_frag(v, ks, db);
          if constexpr (CLEAN) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (!finite(static_cast<float>(a[e]))) a[e] = static_cast<__bf16>(0.f);
          }
          acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc[db], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int row = 8 * (i / 4) + 4 * (lane / 32) + i % 4;
#pragma unroll
        for (int db = 0; db < DP / 32; ++db) {
          const int e = 32 * db + lane % 32;
          float a = *reinterpret_cast<const float*>(v + chunk_at(row, e / 4) + e % 4 * 4);
          if constexpr (CLEAN) a = finite(a) ? a : 0.f;
          acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p[i], acc[db], 0, 0, 0);
        }
      }
    }
  }

  // Whether any of the 32 rows' values is not finite (uniform over the wave).
  static __device__ __forceinline__ bool any_odd(const char* v) {
    const int lane = threadIdx.x % 64;
    bool odd = false;
#pragma unroll 4
    for (int i = 0; i < 32 * kChunks / 64; ++i) {
      const uint4 x = *reinterpret_cast<const uint4*>(v + (i * 64 + lane) * 16);
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        odd |= (w[e] & 0x7f800000u) == 0x7f800000u;
        if constexpr (kBf16) odd |= (w[e] & 0x7f80u) == 0x7f80u;
      }
    }
    return __any(odd);
  }

  // The products of values that are not finite with the weights of the
  // queries that see them; a matrix instruction would multiply them with the
  // zero weights of the others too.  `m2` is the queries' reference of the
  // exponentials, [lo, hi) what they see, j0 the tile's first slot.  Rare: a
  // slot at a time, the score formed again.
  static __device__ __forceinline__ void add_odd_values(const AttnArgs& a, const char* k,
                                                        const char* v, const uint4 (&q)[kQ],
                                                        float m2, int lo, int hi, int j0,
                                                        f32x16 (&acc)[DP / 32]) {
    const int lane = threadIdx.x % 64, h = lane / 32;
    constexpr int per = 16 / sizeof(T);
#pragma unroll 1
    for (int r = 0; r < 32; ++r) {
      float x = 0.f;
#pragma unroll
      for (int i = 0; i < kQ; ++i) {
        const uint4 y = *reinterpret_cast<const uint4*>(k + chunk_at(r, 2 * i + h));
        const uint32_t kw[4] = {y.x, y.y, y.z, y.w}, qw[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (kBf16)
            x += __uint_as_float(kw[e] << 16) * __uint_as_float(qw[e] << 16) +
                 __uint_as_float(kw[e] & 0xffff0000u) * __uint_as_float(qw[e] & 0xffff0000u);
          else
            x += __uint_as_float(kw[e]) * __uint_as_float(qw[e]);
        }
      }
      const float s = score2(a, half_sum(x));
      // a seen slot's weight is positive, however small
      const float p = fmaxf(__builtin_amdgcn_exp2f(s - (m2 == -INFINITY ? 0.f : m2)), 1e-30f);
      const bool sees = j0 + r >= lo && j0 + r < hi;
#pragma unroll
      for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int e = 32 * db + 8 * (i / 4) + 4 * h + i % 4;
          const float y = load_f32<T>(
              reinterpret_cast<const T*>(v + chunk_at(r, e / per)) + e % per);
          if (sees && !finite(y)) acc[db][i] += s != s ? s : p * y;
        }
    }
  }
};

// Offsets (bytes) of a tile's rows: lane i has row i's.
struct RowOffset {
  uint32_t lo, hi;
};

// The block of a tile's row, one row per lane: slot j, clamped to [lo, hi).
__device__ __forceinline__ int row_block(const CacheArgs& c, int b, int j, int lo, int hi) {
  return cache_block(c, b, min(max(j, lo), hi - 1));
}

template <typename T>
__device__ __forceinline__ RowOffset row_offset(const CacheArgs& c, int block, int j, int lo,
                                                int hi) {
  const int64_t o = cache_offset(c, block, min(max(j, lo), hi - 1)) * static_cast<int64_t>(sizeof(T));
  return RowOffset{static_cast<uint32_t>(o), static_cast<uint32_t>(static_cast<uint64_t>(o) >> 32)};
}

// Copies instruction g's rows (g * kRowsPerCopy on) of a tile into LDS at dst:
// 16 bytes per lane, lane-linear, so the lane picks the chunk that belongs at
// its place.  UNIFORM: the rows lie in one block, at the cache's row stride.
template <typename T, int DP, bool UNIFORM>
__device__ __forceinline__ void copy_rows(const char* base, const RowOffset& off, int g,
                                          int64_t row_stride, int d, lds_char* dst) {
  using L = Tile<T, DP>;
  const int lane = threadIdx.x % 64;
  const int sub = lane / L::kChunks, row = g * L::kRowsPerCopy + sub;
  const int c = (lane % L::kChunks) ^ (row & L::kSwz);
  const char* p;
  if constexpr (UNIFORM) {
    const uint32_t lo = __builtin_amdgcn_readlane(off.lo, g * L::kRowsPerCopy);
    const uint32_t hi = __builtin_amdgcn_readlane(off.hi, g * L::kRowsPerCopy);
    p = base + (static_cast<uint64_t>(hi) << 32 | lo) + (sub * static_cast<uint32_t>(row_stride) + c * 16);
  } else {
    const uint32_t lo = __shfl(off.lo, row), hi = __shfl(off.hi, row);
    p = base + (static_cast<uint64_t>(hi) << 32 | lo) + c * 16;
  }
  if (c * 16 < d * static_cast<int>(sizeof(T)))
    __builtin_amdgcn_global_load_lds(p, dst + g * 1024, 16, 0, 0);
}

// Running softmax of a wave's 32 query rows: reference m2 (log2 units; -inf:
// nothing seen yet), sum l of the lane's own slots.
struct Softmax {
  float m2 = -INFINITY, l = 0.f;
};

// One step over NS groups of 32 slots' scores, which become weights; c brings
// them to log2 units.  The reference moves only when a score exceeds it by
// more than 2^8, so the products are rescaled rarely; weights stay below 2^8.
template <int NS, int NB>
__device__ __forceinline__ void softmax_step(float c, f32x16 (&s)[NS], Softmax& st,
                                             f32x16 (&acc)[NB]) {
  float top = s[0][0];
#pragma unroll
  for (int t = 0; t < NS; ++t)
#pragma unroll
    for (int v = t ? 0 : 1; v < 16; ++v) top = fmaxf(top, s[t][v]);
  top = half_max(top) * c;
  if (__any(top - st.m2 > 8.f)) {
    const float m = fmaxf(st.m2, top);
    const float alpha = m == st.m2 ? 1.f : __builtin_amdgcn_exp2f(st.m2 - m);
    st.m2 = m;
    st.l *= alpha;
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[db][v] *= alpha;
  }
  const float ref = st.m2 == -INFINITY ? 0.f : -st.m2;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int t = 0; t < NS; ++t)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      s[t][v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][v], c, ref));
      sum[v % 4] += s[t][v];
    }
  st.l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// Capped scores, in log2 units.
template <int NS>
__device__ __forceinline__ void cap_scores(const AttnArgs& a, f32x16 (&s)[NS]) {
#pragma unroll
  for (int t = 0; t < NS; ++t)
#pragma unroll
    for (int v = 0; v < 16; ++v) s[t][v] = score2(a, s[t][v]);
}

// Scores of slots that query lane n does not see (outside [lo, hi)) become
// -inf; j0 is the slot of the tile's first row.
__device__ __forceinline__ void mask_scores(f32x16& s, int j0, int lo, int hi) {
  const int h = (threadIdx.x % 64) / 32;
  const uint32_t len = static_cast<uint32_t>(max(hi - lo, 0));
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int j = j0 + 8 * (v / 4) + 4 * h + v % 4;
    if (static_cast<uint32_t>(j - lo) >= len) s[v] = -INFINITY;
  }
}

}  // namespace kvx
