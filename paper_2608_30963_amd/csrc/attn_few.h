// attn_few.h -- attention of up to 16 query rows of a KV head under a view:
// single tokens of most models.
//
// As single tokens' kernel (attn_forward_kernels.h), with 16 x 16 matrix
// instructions: half of its sums, scores and weights, so that twice the waves
// fit a compute unit.  Lane (n, g) = (lane % 16, lane / 16) holds query n's
// scores of slots 16 u + 4 g + v (register v of block u), which are the weights'
// operand as they stand if the contraction over 32 slots takes them in that
// order, and columns 16 db + 4 g + v of its sum.  Bound by memory: codes become
// bf16 operands in registers, once a number.  Measured, kernel alone: 64 contexts of
// up to 8k slots in int8, heads 28 / 4 x 128, 307 MB in 71 us, 4.3 TB/s (the ring of 32
// rows: 139); one of 128k 37; 16 of up to 8k slots in bf16 through a window of 1024 with
// sinks, heads 8 / 4 x 256, 67 MB in 19 us (61), of which start and end are 8.
// With the join: 64 contexts of up to 8k slots, heads 8 / 4 x 256, int8 143 us, e4m3 139,
// 4.6 TB/s (174 where registers of e4m3 were kept in scratch memory).
#pragma once

#include "attn_forward.h"
#include "attn_view_tile.h"

namespace kvx {
namespace {

// The values of x over the lanes of a query.
__device__ __forceinline__ void both_rows(float x, float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}
__device__ __forceinline__ float query_max(float x) {
  float a, b;
  both_rows(x, a, b);
  return half_max(fmaxf(a, b));
}
__device__ __forceinline__ float query_sum(float x) {
  float a, b;
  both_rows(x, a, b);
  return half_sum(a + b);
}

// The lane, formed anew: the compiler does not take what derives from it out of a
// loop, where that would fill registers, be kept in scratch memory and be read back,
// for which it waits, and so for every copy in flight.
__device__ __forceinline__ int fresh_lane() {
  int lane;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(lane));
  return lane;
}

// A tile of 32 slots in LDS, rows of DP numbers of S.  16-byte chunk c of row r
// lies at c ^ swz(r), so that the 16 rows of a chunk (keys), or the rows that half
// a wave's transposing read takes (values), cover all of the LDS's 64 banks.
template <typename S, int DP>
struct FewTile {
  static constexpr bool kCoded = sizeof(S) == 1;
  static constexpr int kElem = sizeof(S), kRowBytes = DP * kElem, kChunks = kRowBytes / 16;
  static constexpr int kRowsPerCopy = 64 / kChunks, kBytes = 32 * kRowBytes, kCopies = kBytes / 1024;
  static constexpr int kQ = DP / 32;  // operands of a query
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

  static __device__ __forceinline__ constexpr int key_swz(int r) {
    return kChunks == 4 ? (r >> 2) & 3 : kChunks == 8 ? (r >> 1) & 7 : r & 15;
  }
  static __device__ __forceinline__ constexpr int value_swz(int r) {
    if constexpr (!kCoded) return kChunks == 8 ? (r >> 1 & 3) << 1 : (r & 7) << 1;
    return kChunks == 4   ? (r >> 2 & 1) | (r >> 4 & 1) << 1
           : kChunks == 8 ? (r >> 1 & 3) | (r >> 4 & 1) << 2
                          : (r & 7) | (r >> 4 & 1) << 3;
  }

  struct LaneAt {
    int k;  // keys: row 16 u + n, chunk 4 x + g is at (k ^ 64 x) + 16 u rows
    int v;  // values: column block db at v ^ 32 db (codes: 16 db), + 16 u rows
  };
  static __device__ __forceinline__ LaneAt lane_at() {
    const int lane = threadIdx.x % 64, i = lane % 16, g = lane / 16;
    LaneAt at;
    at.k = i * kRowBytes + (g ^ key_swz(i)) * 16;
    if constexpr (kCoded) {  // 8 rows x 16 codes: 4 g + 0..3 and 16 rows on
      const int row = 4 * g + i / 2 % 4 + 16 * (i / 8);
      at.v = row * kRowBytes + value_swz(row) * 16 + i % 2 * 8;
    } else {  // 4 rows x 16 numbers
      const int row = 4 * g + i / 4;
      at.v = row * kRowBytes + (i % 4 / 2 ^ value_swz(row)) * 16 + i % 2 * 8;
    }
    return at;
  }

  // The query operands of lane (n, g): columns 32 x + 8 g + 0..7 (codes, which a
  // lane reads 16 at a time: 64 (x / 2) + 16 g + 8 (x % 2) + 0..7).
  static __device__ __forceinline__ void load_q(uint4 (&q)[kQ], const bf16_t* row, int d) {
    const int g = threadIdx.x % 64 / 16;
#pragma unroll
    for (int x = 0; x < kQ; ++x) {
      const int e = kCoded ? x / 2 * 64 + g * 16 + x % 2 * 8 : x * 32 + g * 8;
      q[x] = row && e < d ? *reinterpret_cast<const uint4*>(row + e) : uint4{0, 0, 0, 0};
    }
  }

  // Dot products of the 32 rows with the queries, keys times `scale` (e4m3: of rows
  // n and 16 + n; others: 1).
  static __device__ __forceinline__ void scores(f32x4 (&s)[2], const char* k, const LaneAt& at,
                                                const uint4 (&q)[kQ], const float (&scale)[2]) {
    constexpr int kReads = kCoded ? kQ / 2 : kQ;
    uint4 piece[2][kReads];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int x = 0; x < kReads; ++x)
        piece[u][x] = *reinterpret_cast<const uint4*>(k + (at.k ^ 64 * x) + u * 16 * kRowBytes);
#pragma unroll
    for (int u = 0; u < 2; ++u) s[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < kQ; ++x)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        bf16x8 a;
        if constexpr (kCoded) {
          const uint4 p = piece[u][x / 2];
          a = x % 2 ? code_numbers<S>(p.z, p.w, scale[u]) : code_numbers<S>(p.x, p.y, scale[u]);
        } else {
          a = __builtin_bit_cast(bf16x8, piece[u][x]);
        }
        s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, q[x]), s[u], 0, 0, 0);
      }
  }

  // The values' operand of columns 16 db + 0..15, as it is read.
  struct Raw {
    i32x2 x[kCoded ? 1 : 2];
  };
  static __device__ __forceinline__ Raw value_raw(const char* v, const LaneAt& at, int db) {
    Raw r;
    if constexpr (kCoded) {
      r.x[0] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(v + (at.v ^ 16 * db)));
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u)
        r.x[u] = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                               (lds_s16x4*)(v + (at.v ^ 32 * db) + u * 16 * kRowBytes)));
    }
    return r;
  }
  static __device__ __forceinline__ bf16x8 value_numbers(const Raw& r) {
    if constexpr (kCoded) {
      return code_numbers<S>(r.x[0][0], r.x[0][1]);
    } else {
      union {
        i32x2 i[2];
        bf16x8 x;
      } u;
      u.i[0] = r.x[0];
      u.i[1] = r.x[1];
      return u.x;
    }
  }

  // Whether any of the 32 rows' values is not finite (bit 0), and of a row whose
  // bit is set in `rows` (bit 1).  An exponent of ones (a code's seven low bits)
  // passes into the bit above it by one more.
  static __device__ __forceinline__ int odd_values(const char* v, uint32_t rows) {
    if constexpr (std::is_same<S, code_i8>::value) return 0;
    const uint32_t ones = kCoded ? 0x7f7f7f7fu : 0x7f807f80u, more = kCoded ? 0x01010101u : 0x00800080u;
    const int lane = fresh_lane();
    uint32_t any = 0, seen = 0;
#pragma unroll
    for (int i = 0; i < 32 * kChunks / 64; ++i) {
      const int place = i * 64 + lane;
      const uint4 x = *reinterpret_cast<const uint4*>(v + place * 16);
      const uint32_t y = ((x.x & ones) + more) | ((x.y & ones) + more) | ((x.z & ones) + more) | ((x.w & ones) + more);
      any |= y;
      seen |= rows >> place / kChunks & 1 ? y : 0;
    }
    const uint32_t top = kCoded ? 0x80808080u : 0x80008000u;
    return (__any(any & top) ? 1 : 0) | (__any(seen & top) ? 2 : 0);
  }

  // Values that are not finite become zero, in place: products of their own for
  // them would keep a second set of sums.
  static __device__ __forceinline__ void clear_odd_values(char* v) {
    const uint32_t ones = kCoded ? 0x7f7f7f7fu : 0x7f807f80u, more = kCoded ? 0x01010101u : 0x00800080u;
    const uint32_t top = kCoded ? 0x80808080u : 0x80008000u;
    const int lane = threadIdx.x % 64;
    auto clear = [&](uint32_t w) {
      const uint32_t m = ((w & ones) + more) & top;
      return w & ~(kCoded ? (m >> 7) * 0xffu : (m >> 15) * 0xffffu);
    };
#pragma unroll 1
    for (int i = 0; i < 32 * kChunks / 64; ++i) {
      uint4* const at = reinterpret_cast<uint4*>(v + (i * 64 + lane) * 16);
      const uint4 x = *at;
      *at = uint4{clear(x.x), clear(x.y), clear(x.z), clear(x.w)};
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
};

// Whether the 32 slots from j0 on are copied in two runs of 16, each in one block:
// slots of a run that the unit does not see come along, as whatever they hold.
__device__ __forceinline__ bool by_sixteen(const CacheArgs& c, int last) {
  return c.run >= 16 && (c.table || last + 16 <= c.capacity);
}

// Copies 32 rows into LDS at `to`: keys, or values, of the head at `from`, in runs
// from slots first[0] and first[1] on, in blocks id, or (runs false) of slots j0 ..
// j0 + 31, the nearest seen ones instead of those that the unit does not see.
template <typename L, bool KEYS>
__device__ __forceinline__ void few_copy(const CacheArgs& c, const char* from, int b, bool runs, const int (&first)[2],
                                         const int (&id)[2], int j0, const ViewReach& range, int d, uint32_t to) {
  constexpr int R = L::kRowsPerCopy, kHalf = L::kCopies / 2;  // copies of 16 rows
  const int lane = fresh_lane(), sub = lane / L::kChunks, bytes = d * L::kElem;
  auto swz = [](int r) { return KEYS ? L::key_swz(r) : L::value_swz(r); };
  const int chunk = (lane % L::kChunks ^ swz(sub)) * 16;
  const uint32_t st = static_cast<uint32_t>(c.st) * L::kElem;
  if (runs) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int j = first[u];
      const uint32_t slot = c.table ? j - fdiv(c.bs, j) * c.bs.d : j;
      const char* at = from + (c.table ? id[u] : b) * (c.sb * L::kElem) + static_cast<int64_t>(static_cast<uint64_t>(slot) * st);
      if (bytes == L::kRowBytes) {
        uint32_t off[kHalf];
#pragma unroll
        for (int i = 0; i < kHalf; ++i) off[i] = (i * R + sub) * st + (chunk ^ swz(16 * u + i * R) * 16);
        copy16_run<kHalf, 1024>(at, off, to + u * kHalf * 1024);
      } else {
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
          const int e = chunk ^ swz(16 * u + i * R) * 16;
          if (e < bytes) copy16(at, (i * R + sub) * st + e, to + (u * kHalf + i) * 1024);
        }
      }
    }
  } else {
    // lane i finds row i's place
    const int j = range.nearest(j0 + lane % 32);
    const int64_t at = cache_offset(c, cache_block(c, b, j), j) * L::kElem;
    const uint32_t at_lo = static_cast<uint32_t>(at), at_hi = static_cast<uint32_t>(at >> 32);
    // here, and wherever a branch loads: left to itself the compiler waits for the
    // load, and so for all copies, where the branches meet
    __builtin_amdgcn_s_waitcnt(0);
#pragma unroll 1
    for (int i = 0; i < L::kCopies; ++i) {
      const int row = i * R + sub, e = chunk ^ swz(i * R) * 16;
      const int64_t o = static_cast<int64_t>(static_cast<uint64_t>(__shfl(at_hi, row)) << 32 | __shfl(at_lo, row));
      if (e < bytes) copy16(from + o + e, to + i * 1024);
    }
  }
}

template <typename S, int DP>
struct Few {
  using L = FewTile<S, DP>;
  static constexpr int kStage = 2 * L::kBytes + (L::kCoded ? 128 : 0);  // and pairs of scales
  static constexpr int kWaves = 4, kGroups = few_groups(DP, sizeof(S));
  static constexpr int kRoom = 160 * 1024 / kGroups / kWaves / kStage;
  static constexpr int kStages = kRoom < 4 ? kRoom : 4;
  static constexpr int kRing = kStages * kStage;
  static constexpr int kStep = kWaves * 32;  // slots of a workgroup's step
  static_assert(kStages >= 1 && kWaves * kRing * kGroups <= 160 * 1024 && kRing >= kFewRows * DP * 4 + 128, "");
};

template <typename S, int DP>
__device__ __forceinline__ int few_steps(const AttnView& a, const Context& c, int qt) {
  const int r0 = qt * kFewRows;
  const ViewLine<32> line(reach(a, c, r0, min(r0 + kFewRows, c.m * a.group) - 1));
  return max(1, (line.count + Few<S, DP>::kWaves - 1) / Few<S, DP>::kWaves);
}

// A workgroup's equal range of the line, as line_share's; sums over the lanes, and
// the divisions of all but the largest calls, in 32 bits.
template <typename Steps>
__device__ __forceinline__ Share few_share(const AttnView& a, Steps steps_of) {
  const int lane = threadIdx.x % 64;
  int64_t line = 0;
  int mine = 0, upto = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    mine = b0 + lane < a.batch ? steps_of(b0 + lane) : 0;
    upto = a.batch == 1 ? __builtin_amdgcn_readfirstlane(mine) : lanes_upto(mine);
    line += __builtin_amdgcn_readlane(upto, 63);
  }
  Share sh{};
  const int64_t whole = line * a.hkv;
  const bool small = whole <= INT32_MAX;
  sh.per = small ? (static_cast<uint32_t>(whole) + gridDim.x - 1) / gridDim.x : (whole + gridDim.x - 1) / gridDim.x;
  sh.s0 = min<int64_t>(whole, blockIdx.x * sh.per);
  sh.s1 = min(whole, sh.s0 + sh.per);
  if (sh.s0 >= sh.s1) return sh;
  sh.h = small ? static_cast<uint32_t>(sh.s0) / static_cast<uint32_t>(line) : static_cast<int>(sh.s0 / line);
  int64_t into = sh.s0 - sh.h * line;
  for (int b0 = 0;; b0 += 64) {
    if (a.batch > 64) {
      mine = b0 + lane < a.batch ? steps_of(b0 + lane) : 0;
      upto = lanes_upto(mine);
    }
    const uint64_t past = __ballot(upto > into);
    if (past) {
      const int f = __ffsll(static_cast<unsigned long long>(past)) - 1;
      sh.b = b0 + f;
      sh.step = static_cast<int>(into) - (__builtin_amdgcn_readlane(upto, f) - __builtin_amdgcn_readlane(mine, f));
      return sh;
    }
    into -= __builtin_amdgcn_readlane(upto, 63);
  }
}

template <typename S, int DP, Cap CAP>
__global__ void __launch_bounds__((64 * Few<S, DP>::kWaves), (Few<S, DP>::kGroups)) forward_few(AttnView a, ForwardPlan fp) {
  using L = FewTile<S, DP>;
  using F = Few<S, DP>;
  constexpr bool kI8 = std::is_same<S, code_i8>::value;
  constexpr int NW = F::kWaves, NT = 64 * NW, NST = F::kStages, NB = DP / 16;
  __shared__ __attribute__((aligned(16))) char lds[NW * F::kRing];
  const int tid = threadIdx.x, lane = tid % 64, n = lane % 16, g = lane / 16;
  const int w = __builtin_amdgcn_readfirstlane(tid / 64);
  JoinHead* head = fp.heads + blockIdx.x;

  // a unit is one step of the line where units are not split
  const bool whole = fp.splits == 1;
  const Share share = few_share(a, [&](int b) {
    const Context c = context(a, b);
    const int qts = (c.m * a.group + kFewRows - 1) / kFewRows;
    if (whole) return qts;
    int s = 0;
    for (int qt = 0; qt < qts; ++qt) s += few_steps<S, DP>(a, c, qt);
    return s;
  });
  if (tid == 0 && !whole) head->pieces = 0;
  const int64_t s0 = share.s0, s1 = share.s1, per = share.per;
  if (s0 >= s1) return;
  int h = share.h, b = share.b, step = share.step;
  Context c = context(a, b);
  int qt = whole ? step : 0;
  if (whole) step = 0;
  for (int x; step >= (x = few_steps<S, DP>(a, c, qt)); ++qt) step -= x;

  const typename L::LaneAt at = L::lane_at();
  char* const ring = lds + w * F::kRing;
  const uint32_t ring3 = lds_address(lds) + w * F::kRing;

  for (int64_t s = s0; s < s1;) {
    // one unit: steps [step, step + cnt) of its `all`
    const int all = few_steps<S, DP>(a, c, qt);
    const int cnt = whole ? all : static_cast<int>(min<int64_t>(all - step, s1 - s));
    const int r0 = qt * kFewRows, valid = min(kFewRows, c.m * a.group - r0);
    const ViewReach range = reach(a, c, r0, r0 + valid - 1);
    const ViewLine<32> line(range);
    const int tiles = min(cnt, max(line.count - (step * NW + w) + NW - 1, 0) / NW);
    const ViewRow qr = query_row(a, c, r0 + n);
    uint4 q[L::kQ];
    const bf16_t* qp = reinterpret_cast<const bf16_t*>(a.q) + qr.row * a.q_sr + (h * a.group + qr.g) * a.q_sh;
    L::load_q(q, n < valid ? qp : nullptr, a.d);
    const char* kb = a.c.k + h * a.c.sh * static_cast<int64_t>(sizeof(S));
    const char* vb = a.c.v + h * a.c.sh * static_cast<int64_t>(sizeof(S));
    f32x4 acc[NB];
#pragma unroll
    for (int db = 0; db < NB; ++db) acc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    Softmax st;
    __syncthreads();  // LDS is free of the last unit's join
    if (a.d < DP) {
      // copies leave the chunks past head_dim alone: zeros
      for (int i = lane; i < F::kRing / 16; i += 64) reinterpret_cast<uint4*>(ring)[i] = uint4{0, 0, 0, 0};
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }

    auto slot_of = [&](int t) __attribute__((always_inline)) { return line.slot(step * NW + w + t * NW); };
    // A tile's keys (with the scales) and its values are asked for apart, each
    // where the last ones of its stage have been read.  Block numbers: lane i has
    // that of tile base + i / 2 and its slots 16 (i % 2) on: one load for 32 tiles
    // (scalar loads for each would be waited for with the next reads of LDS: 64
    // contexts of up to 8k slots in blocks of 16 took 6 us more).
    constexpr int kKeys = L::kCopies + (L::kCoded ? 1 : 0), kValues = L::kCopies;
    const bool table = a.c.table && a.c.run >= 16 && tiles > 0;
    auto numbers = [&](int t) __attribute__((always_inline)) {
      const int j = sixteen(range, min(slot_of(t + lane / 2), range.hi - 1 & ~31) + 16 * (lane % 2));
      return a.c.table[static_cast<int64_t>(b) * a.c.max_blocks + fdiv(a.c.bs, j)];
    };
    int base = 0, ids = 0, id[2] = {0, 0}, first[2] = {0, 0};
    if (table) ids = numbers(0);
    bool odd = false, runs = false;
    // the queries and numbers are here: the compiler must not wait for them in
    // the loop, where that would be a wait for all copies
    __builtin_amdgcn_s_waitcnt(0);
#pragma unroll 1
    for (int t = -NST; t < tiles; ++t) {
      const int ahead = t + NST;
      // all has been asked for up to tile t + NST - 1
      const bool more = ahead - 1 < tiles, next = ahead < tiles;
      char* const stage = ring + (t + NST) % NST * F::kStage;
      const int j0 = slot_of(max(t, 0));
      f32x4 sc[2] = {};
      uint32_t pair[2][4] = {}, bits = ~0u;
      bool edge = false;
      if (t >= 0) {
        if (more)
          vm_wait<kValues + (NST - 1) * (kKeys + kValues)>();
        else
          vm_wait<0>();
        float mine[2] = {1.f, 1.f};
        if constexpr (L::kCoded) {
          const uint32_t* p = reinterpret_cast<const uint32_t*>(stage + 2 * L::kBytes);
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            if constexpr (!kI8) mine[u] = key_scale(p[16 * u + n]);
            const uint4 y = *reinterpret_cast<const uint4*>(p + 16 * u + 4 * g);
            pair[u][0] = y.x;
            pair[u][1] = y.y;
            pair[u][2] = y.z;
            pair[u][3] = y.w;
          }
        }
        L::scores(sc, stage, at, q, mine);
        edge = !range.all_see(j0, 32);
        if (edge) {
          bits = seen_bits(qr.s, j0) >> 4 * g;
          __builtin_amdgcn_s_waitcnt(0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (next) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // keys and scales are read
        const int k0 = slot_of(ahead);
        const uint32_t to = ring3 + ahead % NST * F::kStage;
        first[0] = k0;
        first[1] = k0 + 16;
        if (!range.inside(k0, 32)) {
          first[0] = sixteen(range, k0);
          first[1] = sixteen(range, k0 + 16);
        }
        runs = by_sixteen(a.c, max(first[0], first[1]));
        if (table) {
          if (ahead - base >= 32) {
            base = ahead;
            ids = numbers(ahead);
            __builtin_amdgcn_s_waitcnt(0);
          }
          id[0] = __builtin_amdgcn_readlane(ids, 2 * (ahead - base));
          id[1] = __builtin_amdgcn_readlane(ids, 2 * (ahead - base) + 1);
        }
        few_copy<L, true>(a.c, kb, b, runs, first, id, k0, range, a.d, to);
        if constexpr (L::kCoded) {
          const int i = lane % 32;
          int j = i < 16 ? first[0] + i : first[1] + i - 16;
          int32_t block = i < 16 ? id[0] : id[1];
          if (!runs) {
            j = range.nearest(k0 + i);
            block = cache_block(a.c, b, j);
            __builtin_amdgcn_s_waitcnt(0);
          }
          if (!a.c.table) block = b;
          if (lane < 32)
            copy4(reinterpret_cast<const char*>(a.scale.p + scale_offset(a.c, a.scale, block, j) + h * a.scale.sh),
                  to + 2 * L::kBytes);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (t >= 0) {
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            float y = sc[u][x];
            if constexpr (kI8) y *= key_scale(pair[u][x]);
            y = CAP == Cap::none   ? y * a.scale2
                : CAP == Cap::part ? __builtin_fmaf(-2.f * a.cap2, cap_part(a, y), a.cap2)
                                   : a.cap2 * cap_tanh(a, y);
            y = bits >> (16 * u + x) & 1 ? y : -INFINITY;
            sc[u][x] = y;
            top = fmaxf(top, y);
          }
        top = query_max(top);
        if (exceeds(st, top, 8.f)) {
          const float m = fmaxf(st.m2, top);
          const float alpha = m == st.m2 ? 1.f : __builtin_amdgcn_exp2f(st.m2 - m);
          st.m2 = m;
          st.l *= alpha;
#pragma unroll
          for (int db = 0; db < NB; ++db) acc[db] *= alpha;
        }
        const float ref = st.m2 == -INFINITY ? 0.f : st.m2;
        bf16x8 p;
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            float y = __builtin_amdgcn_exp2f(sc[u][x] - ref);
            sum += y;
            if constexpr (L::kCoded) {
              y *= value_scale(pair[u][x]);
              y = bits >> (16 * u + x) & 1 ? y : 0.f;  // not 0 times a NaN
            }
            // rounded once to bf16 for the matrix instruction, with its value's scale
            p[4 * u + x] = static_cast<__bf16>(y);
          }
        st.l += sum;
        __builtin_amdgcn_sched_barrier(0);
        if (next)
          vm_wait<(NST - 1) * (kKeys + kValues) + kKeys>();
        else if (more)
          vm_wait<(NST - 1) * (kKeys + kValues)>();
        else
          vm_wait<0>();
        char* const v = stage + L::kBytes;
        // values that are not finite count as zero; if the unit sees any, rows are
        // computed again
        if (edge) {
          const int strange = L::odd_values(v, reach_bits(range, j0));
          odd |= strange > 1;
          if (__builtin_expect(strange, 0)) L::clear_odd_values(v);
        }
        constexpr int kAhead = NB < 8 ? NB : 8;
        typename L::Raw raw[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) raw[i] = L::value_raw(v, at, i);
#pragma unroll
        for (int db = 0; db < NB; ++db) {
          const bf16x8 x = L::value_numbers(raw[db % kAhead]);
          if (db + kAhead < NB) raw[db % kAhead] = L::value_raw(v, at, db + kAhead);
          acc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, p, acc[db], 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (next)
        few_copy<L, false>(a.c, vb, b, runs, first, id, slot_of(ahead), range, a.d,
                           ring3 + ahead % NST * F::kStage + L::kBytes);
    }

    // the waves' results through LDS: each in its own ring, rows of DP floats,
    // 16-byte pieces swizzled by the row; then (m2, l)
    const float l = query_sum(st.l);
    if (n < valid) {
      float4* o = reinterpret_cast<float4*>(ring) + n * (DP / 4);
#pragma unroll
      for (int db = 0; db < NB; ++db)
        o[(4 * db + g) ^ (n & 7)] = float4{acc[db][0], acc[db][1], acc[db][2], acc[db][3]};
      if (g == 0) reinterpret_cast<float2*>(ring + kFewRows * DP * 4)[n] = float2{st.m2, l};
    }
    if (odd) {
#pragma unroll 1
      for (int r = 0; r < valid; ++r) {
        const ViewRow u = query_row(a, c, r0 + r);
        float o[DP / 64];
        Softmax sm;
        const bf16_t* qu = reinterpret_cast<const bf16_t*>(a.q) + u.row * a.q_sr + (h * a.group + u.g) * a.q_sh;
        if (!careful_row<S, bf16_t, DP>(a, b, h, qu, u.s, tiles, slot_of, sm, o)) continue;
#pragma unroll
        for (int i = 0; i < DP / 64; ++i) {
          const int e = i * 64 + lane;
          reinterpret_cast<float*>(ring)[r * DP + ((e / 4) ^ (r & 7)) * 4 + e % 4] = o[i];
        }
        if (lane == 0) reinterpret_cast<float2*>(ring + kFewRows * DP * 4)[r] = float2{sm.m2, sm.l};
      }
    }
    __syncthreads();
    const bool begins = step == 0, ends = step + cnt == all;
    float* part = fp.pieces + (2 * static_cast<size_t>(blockIdx.x) + (begins ? 1 : 0)) * piece_floats(kFewRows, DP);
    for (int i = tid; i < valid * (DP / 4); i += NT) {
      const int r = i / (DP / 4), e = i % (DP / 4);
      float2 ml[NW];
      float m2 = -INFINITY;
#pragma unroll
      for (int x = 0; x < NW; ++x) {
        ml[x] = reinterpret_cast<const float2*>(lds + x * F::kRing + kFewRows * DP * 4)[r];
        m2 = fmaxf(m2, ml[x].x);
      }
      float lsum = 0.f;
      float4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < NW; ++x) {
        const float f = ml[x].x == m2 ? 1.f : __builtin_amdgcn_exp2f(ml[x].x - m2);
        const float4 y = reinterpret_cast<const float4*>(lds + x * F::kRing)[r * (DP / 4) + (e ^ (r & 7))];
        lsum += f * ml[x].y;
        o.x += f * y.x;
        o.y += f * y.y;
        o.z += f * y.z;
        o.w += f * y.w;
      }
      if (begins && ends) {
        const ViewRow u = query_row(a, c, r0 + r);
        const bool sees = sees_any(u);
        if (4 * e < a.d) {
          bf16_t* to = reinterpret_cast<bf16_t*>(a.out) + u.row * a.o_sr + (h * a.group + u.g) * a.o_sh + 4 * e;
          const float x[4] = {o.x, o.y, o.z, o.w};
          bf16_t y[4];
#pragma unroll
          for (int z = 0; z < 4; ++z) y[z] = store_cvt<bf16_t>(sees ? x[z] / lsum : 0.f);
          *reinterpret_cast<uint2*>(to) = __builtin_bit_cast(uint2, y);
        }
        if (a.lse && e == 0)
          a.lse[static_cast<int64_t>(u.row) * a.hq + h * a.group + u.g] =
              sees ? (m2 + __builtin_amdgcn_logf(lsum)) * kLn2 : -INFINITY;
      } else {
        reinterpret_cast<float4*>(part + 2 * kFewRows)[i] = o;
        if (e == 0) reinterpret_cast<float2*>(part)[r] = float2{m2, lsum};
      }
    }
    if (begins && !ends && tid == 0) {
      // the unit's other pieces are the first ones of the next workgroups
      const int64_t end = s - step + all;
      *head = JoinHead{static_cast<int32_t>((end - 1) / per - blockIdx.x + 1), valid, c.q0, r0, h,
                       static_cast<int32_t>(2 * blockIdx.x + 1), 0, 0, b};
    }
    s += whole ? 1 : cnt;
    step = 0;
    if (s < s1) {
      // the next q tile, of this context or one with new tokens after it
      ++qt;
      while (qt * kFewRows >= c.m * a.group) {
        qt = 0;
        if (++b == a.batch) {
          b = 0;
          ++h;
        }
        c = context(a, b);
      }
    }
  }
}

}  // namespace
}  // namespace kvx
