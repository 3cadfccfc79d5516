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

// Waits until at most N vector-memory operations of this wave are outstanding.
template <int N>
__device__ __forceinline__ void vm_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N > 63 ? 63 : N) : "memory");
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

// Rows of head_dim DP (padded with zeros past a.d) in LDS.  16-byte chunk c of
// row r lies at chunk c ^ swz(r) of its row, so that the 16 rows (keys), or the
// 4 rows of 64 bytes (values), that a read instruction takes at a time cover
// all of the LDS's 64 banks: with one swizzle by r % 8 for both, reads took 1.6
// (keys) and 1.8 (values) times as long.  A lane's address is one of a few that
// are formed once (LaneAt) and a constant, since the swizzle is within 256
// (keys) or 128 bytes (values).
template <typename T, int DP>
struct Tile {
  static constexpr int kElem = sizeof(T);
  static constexpr int kChunks = DP * sizeof(T) / 16;
  static constexpr int kKeyAt = kChunks < 16 ? 4 : 8;   // addresses of a lane's key pieces
  static constexpr int kRowBytes = DP * sizeof(T);
  static constexpr int kRowsPerCopy = 64 / kChunks;  // rows of one wave's copy instruction
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int kQ = kBf16 ? DP / 16 : DP / 8;  // 16-byte query pieces of a lane

  static __device__ __forceinline__ constexpr int key_swz(int r) {
    return kChunks < 16 ? (r >> 1) & 7 : r & 15;
  }
  static __device__ __forceinline__ constexpr int value_swz(int r) { return (r & 1) << 2 | ((r >> 1) & 3); }

  struct LaneAt {
    int k[kKeyAt];  // keys: row n, chunk 2 i + h is at k[i % kKeyAt] + i / kKeyAt * kKeyAt * 32
    int v[4];  // values: see value_frag (bf16: two) and add_values
  };
  static __device__ __forceinline__ LaneAt lane_at() {
    const int lane = threadIdx.x % 64, n = lane % 32, h = lane / 32, i = lane % 16;
    LaneAt at;
#pragma unroll
    for (int x = 0; x < kKeyAt; ++x) at.k[x] = n * kRowBytes + ((2 * x + h) ^ key_swz(n)) * 16;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      if constexpr (kBf16) {
        const int row = 4 * h + i / 4, c = 4 * (x & 1) + 2 * (lane / 16 % 2) + i % 4 / 2;
        at.v[x] = row * kRowBytes + (c ^ value_swz(row)) * 16 + i % 2 * 8;
      } else {
        const int row = 4 * h + x;
        at.v[x] = row * kRowBytes + (n / 4 ^ value_swz(row)) * 16 + n % 4 * 4;
      }
    }
    return at;
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

  // Products of the 32 rows at LDS address k with the lanes' row pieces q:
  // lane (n, h) gets its row n's with rows 8 (v / 4) + 4 h + v % 4.  SWAP: its
  // LDS row n's with the pieces' rows.
  template <bool SWAP = false, int AHEAD = 8>
  static __device__ __forceinline__ f32x16 scores(const char* k, const LaneAt& at, const uint4 (&q)[kQ]) {
    // pieces are read AHEAD matrix instructions before their use: the compiler
    // alone reads them just before it and waits
    constexpr int kAhead = kQ < AHEAD ? kQ : AHEAD;
    uint4 piece[kAhead];
    auto read = [&](int i) __attribute__((always_inline)) {
      piece[i % kAhead] =
          *reinterpret_cast<const uint4*>(k + at.k[i % kKeyAt] + i / kKeyAt * kKeyAt * 32);
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) read(i);
    f32x16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
    for (int i = 0; i < kQ; ++i) {
      const uint4 x = piece[i % kAhead];
      if constexpr (kBf16) {
        const bf16x8 a = __builtin_bit_cast(bf16x8, x), b = __builtin_bit_cast(bf16x8, q[i]);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(SWAP ? b : a, SWAP ? a : b, s, 0, 0, 0);
      } else {
        const f32x4 a = __builtin_bit_cast(f32x4, x), b = __builtin_bit_cast(f32x4, q[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s = __builtin_amdgcn_mfma_f32_32x32x2f32(SWAP ? b[e] : a[e], SWAP ? a[e] : b[e], s, 0, 0, 0);
      }
      if (i + kAhead < kQ) read(i + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
    return s;
  }

  // The values' operand of 16 slots (k-step ks of the tile) and 32 columns
  // (block db): lane (m, h) holds column 32 db + m of slots 16 ks + 4 h + 0..3
  // and 16 ks + 8 + 4 h + 0..3.  The transposing read hands lane i of 16 the
  // i-th column of the 4 rows whose 16 columns the lanes' addresses name.
  static __device__ __forceinline__ bf16x8 value_frag(const char* v, const LaneAt& at, int ks, int db) {
    s16x4 r[2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
      r[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_s16x4*)(v + at.v[db % 2] + (16 * ks + 8 * e) * kRowBytes + db / 2 * 128));
    union {
      s16x4 s[2];
      bf16x8 b;
    } u;
    u.s[0] = r[0];
    u.s[1] = r[1];
    return u.b;
  }

  // acc += P V over the tile's 32 slots; CLEAN: values that are not finite
  // count as zero.
  template <bool CLEAN>
  static __device__ __forceinline__ void add_values(const char* v, const LaneAt& at, const f32x16& p,
                                                    f32x16 (&acc)[DP / 32]) {
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
          bf16x8 a = value_frag(v, at, ks, db);
          if constexpr (CLEAN) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (!finite(static_cast<float>(a[e]))) a[e] = static_cast<__bf16>(0.f);
            __builtin_amdgcn_sched_barrier(0);  // rare: few registers rather than speed
          }
          acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc[db], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
#pragma unroll
        for (int db = 0; db < DP / 32; ++db) {
          float a = *reinterpret_cast<const float*>(v + at.v[i % 4] + 8 * (i / 4) * kRowBytes + db * 128);
          if constexpr (CLEAN) a = finite(a) ? a : 0.f;
          acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p[i], acc[db], 0, 0, 0);
        }
      }
    }
  }

  // Whether any of 32 rows' values is not finite (uniform over the wave).  The
  // matrix instructions multiply a value with the zero weights of the queries
  // that do not see it too, so a tile with hidden slots leaves it out, and rows
  // that see it are computed again (careful_row).
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
};

// The LDS address of a shared array, as M0 takes it.
__device__ __forceinline__ uint32_t lds_address(const char* p) {
  return __builtin_amdgcn_readfirstlane(
      static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_char*)(p))));
}

// Copies 16 bytes per lane from global memory into LDS: lane i's go to
// lds + 16 i.  Written out, because the compiler would make every LDS read
// wait for all copies in flight; its own waits for loads only grow by what it
// does not count.  Nothing else here uses M0.  The base is scalar; the no-ops are the wait states between
// a write of M0, or of an SGPR by a vector instruction, and its use.
__device__ __forceinline__ void copy16(const char* from, uint32_t offset, uint32_t lds) {
  const uint64_t p = reinterpret_cast<uint64_t>(from);
  const uint64_t base = static_cast<uint64_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p >> 32))) << 32 |
                        static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p)));
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(lds)),
               "v"(offset), "s"(base)
               : "memory", "m0");
}
__device__ __forceinline__ void copy16(const char* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds)),
               "v"(from)
               : "memory", "m0");
}

// N such copies of one base, to lds + i * STEP: the wait states are spent once.
template <int N, int STEP>
__device__ __forceinline__ void copy16_run(const char* from, const uint32_t* off, uint32_t lds) {
  static_assert(N <= 2 || N % 4 == 0, "");
  const uint64_t p = reinterpret_cast<uint64_t>(from);
  const uint64_t base = static_cast<uint64_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p >> 32))) << 32 |
                        static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p)));
  lds = __builtin_amdgcn_readfirstlane(lds);
  if constexpr (N == 1) {
    copy16(from, off[0], lds);
  } else if constexpr (N == 2) {
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %3\n\t"
        "s_add_u32 m0, m0, %4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3" ::"s"(lds),
        "v"(off[0]), "v"(off[1]), "s"(base), "n"(STEP)
        : "memory", "m0", "scc");
  } else {
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %5\n\t"
        "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %5\n\t"
        "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %5\n\t"
        "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %5" ::"s"(lds),
        "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base), "n"(STEP)
        : "memory", "m0", "scc");
    if constexpr (N > 4) copy16_run<N - 4, STEP>(from, off + 4, lds + 4 * STEP);
  }
}

// 4 bytes per lane, lane i's to lds + 4 i.
__device__ __forceinline__ void copy4(const char* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dword %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(from)
               : "memory", "m0");
}

// The blocks of a tile's slots, one per 16: read by the scalar unit a tile
// ahead of their use, where 16 slots, from a multiple of 16 on, lie in one
// block.
template <int TK>
struct Blocks {
  int32_t id[TK / 16];
};

template <int TK>
__device__ __forceinline__ void fetch_blocks(const CacheArgs& c, int b, int j0, int hi, Blocks<TK>& out) {
  if (!c.table || c.run < 16) return;
  const __attribute__((address_space(4))) int32_t* t =
      (const __attribute__((address_space(4))) int32_t*)(c.table) +
      static_cast<int64_t>(b) * c.max_blocks;
#pragma unroll
  for (int k = 0; k < TK / 16; ++k) out.id[k] = t[fdiv(c.bs, min(j0 + 16 * k, hi - 1))];
}

// The slots [lo, hi) that a unit sees.
struct Range {
  int lo, hi;
  __device__ __forceinline__ bool inside(int j0, int n) const { return j0 >= lo && j0 + n <= hi; }
  __device__ __forceinline__ int nearest(int j) const { return min(max(j, lo), hi - 1); }
};

// Copies rows j0 .. j0 + TK - 1 of a cache (keys at kb, values at vb of one
// head) into LDS at lk and lv, each wave w of WAVES its share, each lane the
// chunk that belongs at its place (L: the rows' layout).  Slots that the unit
// does not see are replaced by the nearest that it does.
template <typename L, int TK, int WAVES, bool KEYS, bool VALUES, typename R_>
__device__ __forceinline__ void copy_tile(const CacheArgs& c, const char* kb, const char* vb, int b,
                                          int j0, const R_& range, const Blocks<TK>& blocks, int d, int w,
                                          uint32_t lk, uint32_t lv) {
  constexpr int R = L::kRowsPerCopy;                          // rows of a copy instruction
  constexpr int kCopies = TK * L::kRowBytes / 1024 / WAVES;   // of a wave, keys or values
  constexpr int kStep = WAVES * R;                            // rows from one to the wave's next
  constexpr int kRun = kStep < 16 ? 16 / kStep : 1;           // of them in 16 slots
  int lane = threadIdx.x % 64;
  if constexpr (kCopies > 8) {
    // what copies derive from the lane is formed anew for every tile: the
    // compiler would take all of it out of the caller's loop, keep it in scratch
    // memory and wait for every copy in flight where it reads it back
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(lane));
  }
  const int sub = lane / L::kChunks;
  const uint32_t st = static_cast<uint32_t>(c.st) * L::kElem;
  // copy i moves rows i kStep + w R + sub: the swizzle of its low bits is the
  // lane's, that of the high ones a constant
  const int low = w * R + sub, bytes = d * L::kElem;
  const int ck = ((lane % L::kChunks) ^ L::key_swz(low)) * 16;
  const int cv = ((lane % L::kChunks) ^ L::value_swz(low)) * 16;
  const int64_t sb = c.sb * L::kElem;
  if (kCopies <= 8 && range.inside(j0, TK) && c.run >= TK && bytes == L::kRowBytes) {
    // the whole tile lies in one block, rows have all of DP: one base (not for
    // more copies, whose offsets would fill the registers)
    const int32_t id = c.table ? blocks.id[0] : b;
    const uint32_t slot = c.table ? j0 - fdiv(c.bs, j0) * c.bs.d : j0;
    const int64_t at = id * sb + static_cast<int64_t>(static_cast<uint64_t>(slot + w * R) * st);
    uint32_t off[kCopies];
    if constexpr (KEYS) {
#pragma unroll
      for (int i = 0; i < kCopies; ++i) off[i] = (i * kStep + sub) * st + (ck ^ (L::key_swz(i * kStep) * 16));
      copy16_run<kCopies, WAVES * 1024>(kb + at, off, lk + w * 1024);
    }
    if constexpr (VALUES) {
#pragma unroll
      for (int i = 0; i < kCopies; ++i) off[i] = (i * kStep + sub) * st + (cv ^ (L::value_swz(i * kStep) * 16));
      copy16_run<kCopies, WAVES * 1024>(vb + at, off, lv + w * 1024);
    }
  } else if (range.inside(j0, TK) && c.run >= 16) {
#pragma unroll
    for (int i = 0; i < kCopies; i += kRun) {
      const int row = i * kStep + w * R, j = j0 + row;  // the first of kRun copies in one block
      int32_t id = b;
      uint32_t slot = j;
      if (c.table) {
        id = blocks.id[i * kStep / 16];
#pragma unroll
        for (int x = 1; x < kStep / 16; ++x)
          if (w * R >= 16 * x) id = blocks.id[i * kStep / 16 + x];
        slot = j - fdiv(c.bs, j) * c.bs.d;
      }
      const int64_t at = id * sb + static_cast<int64_t>(static_cast<uint64_t>(slot) * st);
      const uint32_t to = (i * WAVES + w) * 1024;
      if constexpr (kRun > 1) {
        if (bytes == L::kRowBytes) {
          uint32_t off[kRun];
          if constexpr (KEYS) {
#pragma unroll
            for (int x = 0; x < kRun; ++x)
              off[x] = (x * kStep + sub) * st + (ck ^ (L::key_swz((i + x) * kStep) * 16));
            copy16_run<kRun, WAVES * 1024>(kb + at, off, lk + to);
          }
          if constexpr (VALUES) {
#pragma unroll
            for (int x = 0; x < kRun; ++x)
              off[x] = (x * kStep + sub) * st + (cv ^ (L::value_swz((i + x) * kStep) * 16));
            copy16_run<kRun, WAVES * 1024>(vb + at, off, lv + to);
          }
          continue;
        }
      }
#pragma unroll
      for (int x = 0; x < kRun; ++x) {
        const int k = ck ^ (L::key_swz((i + x) * kStep) * 16), v = cv ^ (L::value_swz((i + x) * kStep) * 16);
        if constexpr (KEYS)
          if (k < bytes) copy16(kb + at, (x * kStep + sub) * st + k, lk + to + x * WAVES * 1024);
        if constexpr (VALUES)
          if (v < bytes) copy16(vb + at, (x * kStep + sub) * st + v, lv + to + x * WAVES * 1024);
      }
    }
  } else {
    // lane i finds row i's place
    const int j = range.nearest(j0 + lane % TK);
    const int64_t at = cache_offset(c, cache_block(c, b, j), j) * L::kElem;
    const uint32_t at_lo = static_cast<uint32_t>(at), at_hi = static_cast<uint32_t>(at >> 32);
#pragma unroll 1
    for (int i = 0; i < kCopies; ++i) {
      const int row = i * kStep + low;
      const int k = ck ^ (L::key_swz(i * kStep) * 16), v = cv ^ (L::value_swz(i * kStep) * 16);
      const int64_t o = static_cast<int64_t>(static_cast<uint64_t>(__shfl(at_hi, row)) << 32 |
                                             __shfl(at_lo, row));
      const uint32_t to = (i * WAVES + w) * 1024;
      if constexpr (KEYS)
        if (k < bytes) copy16(kb + o + k, lk + to);
      if constexpr (VALUES)
        if (v < bytes) copy16(vb + o + v, lv + to);
    }
  }
}

template <typename T, int DP, int TK, int WAVES, bool KEYS = true, bool VALUES = true>
__device__ __forceinline__ void copy_tile(const CacheArgs& c, const char* kb, const char* vb, int b,
                                          int j0, int lo, int hi, const Blocks<TK>& blocks, int d, int w,
                                          uint32_t lk, uint32_t lv) {
  copy_tile<Tile<T, DP>, TK, WAVES, KEYS, VALUES>(c, kb, vb, b, j0, Range{lo, hi}, blocks, d, w, lk, lv);
}

// Query rows of a KV head's unit are (new token, head of the group), the group
// fastest: all heads that share a KV head share its tiles.
struct QueryRow {
  int row, g;  // row of the new tokens, head within the group
  int lo, hi;  // slots that it sees; empty past the context's last row
};

__device__ __forceinline__ bool sees_any(const QueryRow& q) { return q.lo < q.hi; }

__device__ __forceinline__ QueryRow query_row(const AttnArgs& a, const Context& c, int r) {
  QueryRow q;
  const int i = fdiv(a.by_group, r);
  q.row = c.q0 + i;
  q.g = r - i * a.group;
  const int p = c.p0 + i;
  q.lo = first_seen(a, p);
  q.hi = r < c.m * a.group ? end_seen(c, p) : 0;
  return q;
}

// Slots that query rows r0 .. r1 of a context see together; lo == hi: none does.
__device__ __forceinline__ void seen_by(const AttnArgs& a, const Context& c, int r0, int r1,
                                        int& lo, int& hi) {
  const int p0 = c.p0 + fdiv(a.by_group, r0), p1 = c.p0 + fdiv(a.by_group, r1);
  hi = end_seen(c, p1);
  lo = min(first_seen(a, max(p0, 0)), hi);
}

// What query rows r0 .. r1 see: [lo, hi) together, [alo, ahi) all of them.
struct Reach : Range {
  int alo, ahi;
  // no row sees any of slots j .. j + n - 1
  __device__ __forceinline__ bool misses(int j, int n) const { return j >= hi || j + n <= lo; }
  __device__ __forceinline__ bool all_see(int j, int n) const { return j >= alo && j + n <= ahi; }
};

__device__ __forceinline__ Reach reach(const AttnArgs& a, const Context& c, int r0, int r1) {
  Reach r;
  int x;
  seen_by(a, c, r0, r1, r.lo, r.hi);
  seen_by(a, c, r0, r0, x, r.ahi);  // the least that any row's end is
  seen_by(a, c, r1, r1, r.alo, x);  // the most that any row's start is
  return r;
}

// A unit's tiles of TK slots, numbered first .. first + count - 1.
template <int TK>
struct Line {
  int first, count;
  __device__ __forceinline__ explicit Line(const Reach& r)
      : first(r.lo / TK), count(r.lo < r.hi ? (r.hi + TK - 1) / TK - r.lo / TK : 0) {}
  __device__ __forceinline__ int slot(int t) const { return t * TK; }
  // the first tile that ends past slot `to`
  __device__ __forceinline__ int until(int to) const { return to / TK; }
};

// Query rows [from, to) of those from r0 on that see anything: slots before them
// are negative, windows after them start past the cache's last slot.
__device__ __forceinline__ void seeing(const AttnArgs& a, const Context& c, int r0, int& from, int& to) {
  from = max(0, -c.p0) * a.group - r0;  // slots times heads may pass 32 bits, rows do not
  const int64_t last = a.window ? min<int64_t>(c.m, int64_t(c.n) + a.window - 1 - c.p0) : c.m;
  to = static_cast<int>(max<int64_t>(last, 0)) * a.group - r0;
}

// A workgroup's equal range of the line (KV head, context, step), where context
// b has steps_of(b) steps.
struct Share {
  int64_t s0, s1;  // of the line; empty: nothing to do
  int64_t per;     // length of every workgroup's range
  int h, b, step;  // where s0 lies
};

// Inclusive sum over a wave's lanes.
__device__ __forceinline__ int64_t wave_sum(int64_t x) {
  const int lane = threadIdx.x % 64;
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) {
    const int64_t y = __shfl_up(x, i);
    if (lane >= i) x += y;
  }
  return x;
}

// Found by every wave for itself, 64 contexts at a time (a launch of few
// contexts waits for no barrier); the waves' results are the same.
template <typename Steps>
__device__ __forceinline__ Share line_share(const AttnArgs& a, Steps steps_of) {
  const int lane = threadIdx.x % 64;
  int64_t line = 0, mine = 0, upto = 0;  // line: of one head
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    mine = b0 + lane < a.batch ? steps_of(b0 + lane) : 0;
    upto = wave_sum(mine);
    line += __shfl(upto, 63);
  }
  Share sh{};
  const int64_t whole = line * a.hkv;
  sh.per = (whole + gridDim.x - 1) / gridDim.x;
  sh.s0 = min<int64_t>(whole, blockIdx.x * sh.per);
  sh.s1 = min(whole, sh.s0 + sh.per);
  if (sh.s0 >= sh.s1) return sh;
  sh.h = __builtin_amdgcn_readfirstlane(static_cast<int>(sh.s0 / line));
  int64_t into = sh.s0 - sh.h * line;
  for (int b0 = 0;; b0 += 64) {
    if (a.batch > 64) {
      mine = b0 + lane < a.batch ? steps_of(b0 + lane) : 0;
      upto = wave_sum(mine);
    }
    const uint64_t past = __ballot(upto > into);
    if (past) {
      const int f = __ffsll(static_cast<unsigned long long>(past)) - 1;
      sh.b = __builtin_amdgcn_readfirstlane(b0 + f);
      sh.step = __builtin_amdgcn_readfirstlane(static_cast<int>(into - (__shfl(upto, f) - __shfl(mine, f))));
      return sh;
    }
    into -= __shfl(upto, 63);
  }
}

// Waves and stages of the rings of 32-slot tiles that a workgroup holds in LDS
// for single tokens, `stage` bytes a tile.
constexpr int ring_waves(int stage) { return stage <= 16384 ? 4 : stage <= 32768 ? 2 : 1; }
constexpr int ring_stages(int stage) {
  const int n = 131072 / ring_waves(stage) / stage;
  return n < 4 ? n : 4;
}

// Running softmax of a wave's 32 query rows: reference m2 (log2 units; -inf:
// nothing seen yet), sum l of the lane's own slots.
struct Softmax {
  float m2 = -INFINITY, l = 0.f;
};

// The largest of a query's scores of NS groups of 32 slots, in log2 units (c
// brings them there).
template <int NS>
__device__ __forceinline__ float top_score(float c, const f32x16 (&s)[NS]) {
  float top = s[0][0];
#pragma unroll
  for (int t = 0; t < NS; ++t)
#pragma unroll
    for (int v = t ? 0 : 1; v < 16; ++v) top = fmaxf(top, s[t][v]);
  return half_max(top) * c;
}

// Whether a score exceeds its query's reference by more than 2^by.
__device__ __forceinline__ bool exceeds(const Softmax& st, float top, float by) {
  return __any(top - st.m2 > by);
}

// How far scores may pass their reference without a rescaling (log2 units).
// Weights and sums are floating-point numbers, as exact at 2^24 as at 1.  What
// bounds it is the sums of values, which grow by the same: values of sum |v| up to
// 2^104 over the slots stay below fp32's largest, 2^128.
constexpr float kRoom = 24.f;

template <int NB>
__device__ __forceinline__ void rescale(Softmax& st, float top, f32x16 (&acc)[NB]) {
  const float m = fmaxf(st.m2, top);
  const float alpha = m == st.m2 ? 1.f : __builtin_amdgcn_exp2f(st.m2 - m);
  st.m2 = m;
  st.l *= alpha;
#pragma unroll
  for (int db = 0; db < NB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] *= alpha;
}

// 32 slots' scores become weights.
__device__ __forceinline__ void weights(float c, f32x16& s, Softmax& st) {
  const float ref = st.m2 == -INFINITY ? 0.f : -st.m2;
  float sum[2] = {0.f, 0.f};
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    s[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v], c, ref));
    sum[v % 2] += s[v];
  }
  st.l += sum[0] + sum[1];
}

template <int NS, int NB>
__device__ __forceinline__ void softmax_step(float c, f32x16 (&s)[NS], Softmax& st,
                                             f32x16 (&acc)[NB]) {
  const float top = top_score(c, s);
  if (exceeds(st, top, 8.f)) rescale(st, top, acc);
#pragma unroll
  for (int t = 0; t < NS; ++t) weights(c, s[t], st);
}

// How attention forms capped scores: bf16 ones, under caps up to kPartCap, by
// cap_part, all others by cap_tanh.  Measured (us, a few calls in a row; cap_part,
// cap_tanh), cap 50: 1531 tokens in 5627 slots, window 4096, heads 8 / 4 x 256: 125,
// 153; 1024 in 8192, heads 28 / 4 x 128: 202, 279; 64 contexts of single tokens over
// up to 8k slots, heads 28 / 4 x 128: 124, 134.
enum class Cap { none, part, tanh };

// Capped scores, in log2 units.
template <Cap CAP, int NS>
__device__ __forceinline__ void cap_scores(const AttnArgs& a, f32x16 (&s)[NS]) {
#pragma unroll
  for (int t = 0; t < NS; ++t)
#pragma unroll
    for (int v = 0; v < 16; ++v)
      s[t][v] = CAP == Cap::part ? __builtin_fmaf(-2.f * a.cap2, cap_part(a, s[t][v]), a.cap2)
                     : a.cap2 * cap_tanh(a, s[t][v]);
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

// A tile of 32 slots that not all of the wave's queries see.  Returns whether
// it holds values that are not finite, which it leaves out.
template <typename T, int DP, Cap CAP>
__device__ __forceinline__ bool edge_step(const AttnArgs& a, const char* k, const char* v,
                                          const typename Tile<T, DP>::LaneAt& at,
                                          const uint4 (&q)[Tile<T, DP>::kQ], int j0, int lo, int hi,
                                          Softmax& st, f32x16 (&acc)[DP / 32]) {
  using L = Tile<T, DP>;
  const bool odd = L::any_odd(v);
  f32x16 s[1] = {L::scores(k, at, q)};
  if constexpr (CAP != Cap::none) cap_scores<CAP>(a, s);
  mask_scores(s[0], j0, lo, hi);
  softmax_step(CAP == Cap::none ? a.scale2 : 1.f, s, st, acc);
  if (odd)
    L::template add_values<true>(v, at, s[0], acc);
  else
    L::template add_values<false>(v, at, s[0], acc);
  return odd;
}

// What the weights and values of one query row give over a list of tiles of 32
// slots, one slot at a time: lane e holds columns e, e + 64, .. of the sum.
// Products with slots that the row does not see are never formed.  `slot(t)`
// is tile t's first slot.  Returns whether a sum is not finite: then the row
// sees such a value, and only then is this its result (a row that does not
// keeps the bits that it has without them).
template <typename T, int DP, typename Slot>
__device__ __forceinline__ bool careful_row(const AttnArgs& a, int b, int h, const T* q, int lo,
                                            int hi, int tiles, Slot slot, Softmax& st,
                                            float (&o)[DP / 64]) {
  const int lane = threadIdx.x % 64, n = lane % 32, half = lane / 32;
  const T* kc = reinterpret_cast<const T*>(a.c.k) + h * a.c.sh;
  const T* vc = reinterpret_cast<const T*>(a.c.v) + h * a.c.sh;
  st = Softmax{};
#pragma unroll
  for (int i = 0; i < DP / 64; ++i) o[i] = 0.f;
#pragma unroll 1
  for (int t = 0; t < tiles; ++t) {
    const int j = slot(t) + n;
    const bool sees = j >= lo && j < hi;
    if (!__any(sees)) continue;
    const int jc = min(max(j, lo), hi - 1);
    const int64_t at = cache_offset(a.c, cache_block(a.c, b, jc), jc);
    float x = 0.f;
#pragma unroll 1
    for (int e = half; e < a.d; e += 2) x += load_f32<T>(q + e) * load_f32<T>(kc + at + e);
    x = half_sum(x);
    const float s = sees ? score2(a, x) : -INFINITY;
    float top = s;
#pragma unroll
    for (int i = 16; i; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
    const float m = fmaxf(st.m2, top);
    const float alpha = m == st.m2 ? 1.f : __builtin_amdgcn_exp2f(st.m2 - m);
    st.m2 = m;
    // a seen slot's weight is positive, however small
    float p = __builtin_amdgcn_exp2f(s - (m == -INFINITY ? 0.f : m));
    if (sees && p == 0.f && s > -INFINITY) p = 1e-30f;
    float sum = p;
#pragma unroll
    for (int i = 16; i; i >>= 1) sum += __shfl_xor(sum, i);
    st.l = st.l * alpha + sum;
#pragma unroll
    for (int i = 0; i < DP / 64; ++i) o[i] *= alpha;
#pragma unroll 1
    for (int r = 0; r < 32; ++r) {
      if (!__shfl(static_cast<int>(sees), r)) continue;
      const float pr = __shfl(p, r);
      const int64_t vr = static_cast<int64_t>(
          static_cast<uint64_t>(__shfl(static_cast<uint32_t>(at >> 32), r)) << 32 |
          __shfl(static_cast<uint32_t>(at), r));
#pragma unroll
      for (int i = 0; i < DP / 64; ++i)
        if (i * 64 + lane < a.d) o[i] += pr * load_f32<T>(vc + vr + i * 64 + lane);
    }
  }
  bool odd = false;
#pragma unroll
  for (int i = 0; i < DP / 64; ++i) odd |= !finite(o[i]);
  return __any(odd);
}

}  // namespace kvx
