// attn_view_tile.h -- what the attention kernels do under a view: masks, tiles
// before and in a window, and tiles of caches of 8 bits.
#pragma once

#include "attn_forward.h"
#include "attn_tile.h"
#include "attn_view.h"

namespace kvx {

// The numbers that a cache of S is computed with.
template <typename S>
struct NumbersOf {
  using type = S;
};
template <>
struct NumbersOf<code_i8> {
  using type = bf16_t;
};
template <>
struct NumbersOf<code_e4m3> {
  using type = bf16_t;
};
template <typename S>
using Numbers = typename NumbersOf<S>::type;

struct ViewRow : QueryRow {
  Sight s;
};

__device__ __forceinline__ bool sees_any(const ViewRow& q) { return sees_any(q.s); }

__device__ __forceinline__ ViewRow query_row(const AttnView& a, const Context& c, int r) {
  ViewRow q;
  const int i = fdiv(a.by_group, r);
  q.row = c.q0 + i;
  q.g = r - i * a.group;
  q.s = Sight{0, 0, 0, c.p0, c.n, 0, nullptr};
  if (r < c.m * a.group) q.s = sight(a, c, i);
  q.lo = q.s.lo;
  q.hi = q.s.hi;
  return q;
}

// The slots that a unit sees: [lo, hi), and those below sink.
struct ViewReach : Reach {
  int sink, all_sink;
  __device__ __forceinline__ bool inside(int j0, int n) const { return Range::inside(j0, n) || j0 + n <= sink; }
  __device__ __forceinline__ int nearest(int j) const {
    return j < sink ? j : lo < hi ? Range::nearest(j) : sink - 1;
  }
  __device__ __forceinline__ bool misses(int j, int n) const { return Reach::misses(j, n) && j >= sink; }
  __device__ __forceinline__ bool all_see(int j, int n) const { return Reach::all_see(j, n) || j + n <= all_sink; }
};

// A tree's nodes are at positions p0 .. p0 + m - 1, in any order.
__device__ __forceinline__ ViewReach reach(const AttnView& a, const Context& c, int r0, int r1) {
  ViewReach r;
  static_cast<Reach&>(r) = reach(static_cast<const AttnArgs&>(a), c, r0, r1);
  if (a.tree) {
    const int i0 = fdiv(a.by_group, r0), i1 = fdiv(a.by_group, r1);
    r.hi = c.p0 + i1 >= 0 ? c.n : 0;
    r.lo = min(first_seen(a, max(c.p0, 0)), r.hi);
    r.ahi = c.p0 + i0 >= 0 ? min(max(c.p0, 0), c.n) : 0;
    r.alo = first_seen(a, max(c.p0 + c.m - 1, 0));
    r.sink = min(a.sink, min(max(c.p0, 0), r.hi));
  } else {
    r.sink = min(a.sink, r.hi);
  }
  r.all_sink = min(a.sink, r.ahi);
  return r;
}

// Which of the slots j0 .. j0 + 31 the unit sees, slot j0 + i in bit i.
__device__ __forceinline__ uint32_t reach_bits(const ViewReach& r, int j0) {
  return low_bits(r.hi - j0) & (~low_bits(r.lo - j0) | low_bits(r.sink - j0));
}

// The 16 slots that are copied for slots j .. j + 15: themselves where the unit
// sees any of them, else those around the nearest that it does.
__device__ __forceinline__ int sixteen(const ViewReach& r, int j) {
  const bool seen = j < r.sink || (j + 16 > r.lo && j < r.hi && r.lo < r.hi);
  return seen ? j : r.nearest(j) & ~15;
}

// A unit's tiles: those of the sinks that lie before the window, then its own.
template <int TK>
struct ViewLine {
  static constexpr int first = 0;
  int before, skip, count;
  __device__ __forceinline__ explicit ViewLine(const ViewReach& r) {
    const int sinks = (r.sink + TK - 1) / TK;
    if (r.lo < r.hi) {
      before = min(sinks, r.lo / TK);
      skip = r.lo / TK - before;
      count = before + (r.hi + TK - 1) / TK - r.lo / TK;
    } else {
      before = count = sinks;
      skip = 0;
    }
  }
  __device__ __forceinline__ int slot(int t) const { return (t < before ? t : t + skip) * TK; }
  __device__ __forceinline__ int until(int to) const { return max(to / TK - skip, 0); }
};

template <int TK, typename A>
struct LineOf {
  using type = Line<TK>;
};
template <int TK>
struct LineOf<TK, AttnView> {
  using type = ViewLine<TK>;
};

// A workgroup's piece of the chunk kernel's work: strips (128 query rows of a KV
// head) are cut into pieces of about the same number of tiles, as many as there
// are workgroups beyond one a strip, by every context's length.  Equal numbers of
// pieces for all took the longest context's time: trees of 64 nodes, 8 contexts
// of 800 to 8k slots, heads 28 / 4 x 128, 120 us.  b < 0: nothing to do.
struct ChunkShare {
  int strips;         // of a head, all contexts'
  int h, b, qt, strip;
  int piece, pieces;  // of the strip
  int first, step;    // index of its first piece, and from one to the next
};

// Inclusive sum over a wave's lanes.
__device__ __forceinline__ int lanes_upto(int x) {
  const int lane = threadIdx.x % 64;
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) {
    const int y = __shfl_up(x, i);
    if (lane >= i) x += y;
  }
  return x;
}

template <int TK>
__device__ __forceinline__ ChunkShare chunk_share(const AttnView& a, bool split) {
  const int lane = threadIdx.x % 64;
  int cnt = 0, tiles = 0;  // strips of the lane's context, and their tiles
  auto look = [&](int b0) __attribute__((always_inline)) {
    cnt = tiles = 0;
    if (b0 + lane < a.batch) {
      const Context c = context(a, b0 + lane);
      const int rows = c.m * a.group;
      cnt = (rows + kChunkRows - 1) / kChunkRows;
      if (split && rows > 0) tiles = ViewLine<TK>(reach(a, c, 0, rows - 1)).count;
    }
  };
  ChunkShare s{};
  s.b = -1;
  // tiles of all strips, not less than they are: 64 bits' worth in fp32
  float all = 0.f;
  int strips = 0, strips_upto = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    look(b0);
    strips_upto = lanes_upto(cnt);
    strips += __builtin_amdgcn_readlane(strips_upto, 63);
    if (split) {
      float x = static_cast<float>(cnt) * static_cast<float>(tiles);
#pragma unroll
      for (int i = 32; i; i >>= 1) x += __shfl_xor(x, i);
      all += x;
    }
  }
  s.strips = strips;
  int per = INT32_MAX, groups = strips, upto = strips_upto;  // groups: workgroups of a head
  auto pieces_of = [&](int t) __attribute__((always_inline)) { return max(1, (t - 1) / per + 1); };
  const int more = static_cast<int>(gridDim.x) - strips * a.hkv;
  if (split && more > 0) {
    // the least tiles a piece that the grid may have room for, somewhat more, and
    // what it has room for: sum of ceil(tiles / per) <= strips + all / per
    all *= a.hkv * 1.0001f;
    for (int turn = 0; turn < 3; ++turn) {
      const float share = turn < 2 ? all / gridDim.x * (turn ? 1.15f : 1.f) : all / more;
      per = __builtin_amdgcn_readfirstlane(static_cast<int>(min(share + 1.f, 1e9f)));
      groups = 0;
      for (int b0 = 0; b0 < a.batch; b0 += 64) {
        if (a.batch > 64) look(b0);
        upto = lanes_upto(cnt * pieces_of(tiles));
        groups += __builtin_amdgcn_readlane(upto, 63);
      }
      if (groups * a.hkv <= static_cast<int>(gridDim.x)) break;
    }
  }
  // consecutive workgroups of an XCD share a head's cache, and a context's tiles;
  // those with nothing to do are the last ones, so that no XCD has more than others
  const int used = groups * a.hkv;
  if (static_cast<int>(blockIdx.x) >= used) return s;
  const int id = xcd_remap(blockIdx.x, used);
  s.h = id / groups;
  int into = id - s.h * groups, before = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    int n = pieces_of(tiles);
    if (a.batch > 64) {
      look(b0);
      n = pieces_of(tiles);
      upto = lanes_upto(cnt * n);
      strips_upto = lanes_upto(cnt);
    }
    const uint64_t past = __ballot(upto > into);
    if (past) {
      const int f = __ffsll(static_cast<unsigned long long>(past)) - 1;
      const int strips_b = __builtin_amdgcn_readlane(cnt, f);
      s.pieces = __builtin_amdgcn_readlane(n, f);
      const int in_context = into - (__builtin_amdgcn_readlane(upto, f) - strips_b * s.pieces);
      s.b = b0 + f;
      s.piece = in_context / strips_b;
      s.qt = strips_b - 1 - in_context % strips_b;  // later strips, which see more, first
      s.strip = before + __builtin_amdgcn_readlane(strips_upto, f) - strips_b + s.qt;
      s.first = id - s.piece * strips_b;
      s.step = strips_b;
      return s;
    }
    into -= __builtin_amdgcn_readlane(upto, 63);
    before += __builtin_amdgcn_readlane(strips_upto, 63);
  }
  return s;
}

// What a lane's query sees of the slots of its 16 scores: bit 8 (v / 4) + v % 4
// stands for register v.
__device__ __forceinline__ uint32_t lane_bits(const Sight& s, int j0) {
  return seen_bits(s, j0) >> (threadIdx.x % 64 / 32 * 4);
}
__device__ __forceinline__ bool lane_sees(uint32_t bits, int v) { return bits >> (8 * (v / 4) + v % 4) & 1; }

__device__ __forceinline__ void mask_scores(f32x16& s, uint32_t bits) {
#pragma unroll
  for (int v = 0; v < 16; ++v)
    if (!lane_sees(bits, v)) s[v] = -INFINITY;
}

// As edge_step.
template <typename T, int DP, Cap CAP>
__device__ __forceinline__ bool edge_step(const AttnView& a, const char* k, const char* v,
                                          const typename Tile<T, DP>::LaneAt& at,
                                          const uint4 (&q)[Tile<T, DP>::kQ], int j0, const Sight& row,
                                          Softmax& st, f32x16 (&acc)[DP / 32]) {
  using L = Tile<T, DP>;
  const bool odd = L::any_odd(v);
  f32x16 s[1] = {L::scores(k, at, q)};
  if constexpr (CAP != Cap::none) cap_scores<CAP>(a, s);
  mask_scores(s[0], lane_bits(row, j0));
  softmax_step(CAP == Cap::none ? a.scale2 : 1.f, s, st, acc);
  if (odd)
    L::template add_values<true>(v, at, s[0], acc);
  else
    L::template add_values<false>(v, at, s[0], acc);
  return odd;
}

// As careful_row, of what the row sees under a view.
template <typename S, typename T, int DP, typename Slot>
__device__ __forceinline__ bool careful_row(const AttnView& a, int b, int h, const T* q, const Sight& row,
                                            int tiles, Slot slot, Softmax& st, float (&o)[DP / 64]) {
  const int lane = threadIdx.x % 64, n = lane % 32, half = lane / 32;
  const S* kc = reinterpret_cast<const S*>(a.c.k) + h * a.c.sh;
  const S* vc = reinterpret_cast<const S*>(a.c.v) + h * a.c.sh;
  st = Softmax{};
#pragma unroll
  for (int i = 0; i < DP / 64; ++i) o[i] = 0.f;
#pragma unroll 1
  for (int t = 0; t < tiles; ++t) {
    const int j0 = slot(t);
    const uint32_t bits = __builtin_amdgcn_readfirstlane(seen_bits(row, j0));
    if (!bits) continue;
    const bool sees = bits >> n & 1;
    const int j = j0 + (sees ? n : __ffs(bits) - 1);
    const int32_t block = cache_block(a.c, b, j);
    const int64_t at = cache_offset(a.c, block, j);
    float kf = 1.f, vf = 1.f;
    if constexpr (sizeof(S) == 1) {
      const uint32_t pair = a.scale.p[scale_offset(a.c, a.scale, block, j) + h * a.scale.sh];
      kf = key_scale(pair);
      vf = value_scale(pair);
    }
    float x = 0.f;
#pragma unroll 1
    for (int e = half; e < a.d; e += 2) x += load_f32<T>(q + e) * number<S>(kc + at + e, 1.f);
    x = half_sum(x) * kf;
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
      if (!(bits >> r & 1)) continue;
      const float pr = __shfl(p, r), f = __shfl(vf, r);
      const int64_t vr = static_cast<int64_t>(
          static_cast<uint64_t>(__shfl(static_cast<uint32_t>(static_cast<uint64_t>(at) >> 32), r)) << 32 |
          __shfl(static_cast<uint32_t>(at), r));
#pragma unroll
      for (int i = 0; i < DP / 64; ++i)
        if (i * 64 + lane < a.d) o[i] += pr * number<S>(vc + vr + i * 64 + lane, f);
    }
  }
  bool odd = false;
#pragma unroll
  for (int i = 0; i < DP / 64; ++i) odd |= !finite(o[i]);
  return __any(odd);
}

// ---------------------------------------------------------------------------
// Codes in LDS
// ---------------------------------------------------------------------------

// Rows of codes as they come, for what turns them into a Tile<bf16_t, DP>.
template <int DP>
struct CodeRows {
  static constexpr int kChunks = DP / 16, kRowsPerCopy = 64 / kChunks;
};

// Rows of codes that operands are read from (as Tile).  A lane reads 16 codes of
// a key at a time, the operands of two matrix instructions, so that the queries'
// operands take the columns in that order too: lane (n, h) has columns 32 s +
// 16 h + 8 e of them in instruction 2 s + e.  Values come by the transposing read
// of 8 rows x 16 codes.  Swizzles let 16 rows of keys, and the 8 rows x 32 codes
// of values that half a wave reads, cover all of the LDS's 64 banks.
template <typename C, int DP>
struct CodeTile {
  static constexpr int kElem = 1, kChunks = DP / 16, kRowBytes = DP, kRowsPerCopy = 64 / kChunks;
  static constexpr int kQ = DP / 16;
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

  static __device__ __forceinline__ constexpr int key_swz(int r) {
    return kChunks == 4 ? (r >> 2) & 3 : kChunks == 8 ? (r >> 1) & 7 : r & 15;
  }
  static __device__ __forceinline__ constexpr int value_swz(int r) {
    return kChunks == 4   ? (r >> 3 & 1) << 1
           : kChunks == 8 ? (r >> 1 & 1) << 1 | (r >> 3 & 1) << 2
                          : (r & 1) << 1 | (r >> 1 & 1) << 2 | (r >> 3 & 1) << 3;
  }

  struct LaneAt {
    int k;  // keys: row n, chunk 2 s + h is at k ^ 32 s
    int v;  // values: column block db, slots 16 ks + .. at (v ^ 32 db) + 16 ks rows
  };
  static __device__ __forceinline__ LaneAt lane_at() {
    const int lane = threadIdx.x % 64, n = lane % 32, h = lane / 32, i = lane % 16;
    const int row = (i / 8) * 8 + 4 * h + i / 2 % 4;
    return LaneAt{n * kRowBytes + (h ^ key_swz(n)) * 16,
                  row * kRowBytes + ((lane / 16 % 2) ^ value_swz(row)) * 16 + i % 2 * 8};
  }

  static __device__ __forceinline__ void load_q(uint4 (&q)[kQ], const bf16_t* row, int d) {
    const int h = (threadIdx.x % 64) / 32;
#pragma unroll
    for (int s = 0; s < kQ; ++s) {
      const int e = s / 2 * 32 + h * 16 + s % 2 * 8;
      q[s] = row && e < d ? *reinterpret_cast<const uint4*>(row + e) : uint4{0, 0, 0, 0};
    }
  }

  // As Tile's, of keys times `scale`, lane (n, h)'s of row n (e4m3; int8: 1).
  static __device__ __forceinline__ f32x16 scores(const char* k, const LaneAt& at, const uint4 (&q)[kQ],
                                                  float scale) {
    uint4 piece[kQ / 2];
#pragma unroll
    for (int s = 0; s < kQ / 2; ++s) piece[s] = *reinterpret_cast<const uint4*>(k + (at.k ^ 32 * s));
    f32x16 x;
#pragma unroll
    for (int v = 0; v < 16; ++v) x[v] = 0.f;
#pragma unroll
    for (int s = 0; s < kQ / 2; ++s) {
      const uint4 p = piece[s];
      x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(code_numbers<C>(p.x, p.y, scale),
                                                  __builtin_bit_cast(bf16x8, q[2 * s]), x, 0, 0, 0);
      x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(code_numbers<C>(p.z, p.w, scale),
                                                  __builtin_bit_cast(bf16x8, q[2 * s + 1]), x, 0, 0, 0);
    }
    return x;
  }

  // The codes of value_frag.
  static __device__ __forceinline__ i32x2 value_codes(const char* v, const LaneAt& at, int ks, int db) {
    return __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(v + (at.v ^ 32 * db) + 16 * ks * kRowBytes));
  }

  // Whether any of 32 rows' codes is no number.
  static __device__ __forceinline__ bool any_odd(const char* v) {
    if constexpr (std::is_same<C, code_i8>::value) return false;
    const int lane = threadIdx.x % 64;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 32 * kChunks / 64; ++i) {
      const uint4 x = *reinterpret_cast<const uint4*>(v + (i * 64 + lane) * 16);
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
      // a byte of which all low seven bits are set passes 127 by one more
#pragma unroll
      for (int e = 0; e < 4; ++e) odd |= ((w[e] & 0x7f7f7f7fu) + 0x01010101u & 0x80808080u) != 0;
    }
    return __any(odd);
  }
};

// Whether values of slots j0 .. j0 + n - 1 that the unit sees are no numbers (n is at
// most a wave's lanes).
template <typename C>
__device__ __forceinline__ bool odd_codes(const AttnView& a, int b, int h, const ViewReach& range, int j0, int n) {
  const int j = j0 + static_cast<int>(threadIdx.x % 64);
  bool odd = false;
  if (j < j0 + n && !range.misses(j, 1)) {
    const int32_t block = cache_block(a.c, b, j);
    odd = !finite(value_scale(a.scale.p[scale_offset(a.c, a.scale, block, j) + h * a.scale.sh]));
    if constexpr (!std::is_same<C, code_i8>::value) {
      const char* v = a.c.v + h * a.c.sh + cache_offset(a.c, block, j);
#pragma unroll 1
      for (int e = 0; e < a.d; e += 16) {
        const uint4 x = *reinterpret_cast<const uint4*>(v + e);
        const uint32_t low = 0x7f7f7f7fu, one = 0x01010101u;  // seven set bits pass into the eighth
        odd |= ((((x.x & low) + one) | ((x.y & low) + one) | ((x.z & low) + one) | ((x.w & low) + one)) & 0x80808080u) != 0;
      }
    }
  }
  return __any(odd);
}

// The tile that single tokens' kernel reads.
template <typename S, int DP>
struct TileOf {
  using type = Tile<S, DP>;
};
template <int DP>
struct TileOf<code_i8, DP> {
  using type = CodeTile<code_i8, DP>;
};
template <int DP>
struct TileOf<code_e4m3, DP> {
  using type = CodeTile<code_e4m3, DP>;
};

// The scales of the slots of a lane's 16 scores, of 32 pairs in LDS.
__device__ __forceinline__ void lane_pairs(const char* pairs, uint32_t (&pair)[16]) {
  const int h = (threadIdx.x % 64) / 32;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const uint4 y = *reinterpret_cast<const uint4*>(pairs + (8 * x + 4 * h) * 4);
    pair[4 * x] = y.x;
    pair[4 * x + 1] = y.y;
    pair[4 * x + 2] = y.z;
    pair[4 * x + 3] = y.w;
  }
}

// A tile of 32 slots of codes at k and v, scale pairs at `pairs`.  EDGE: not all
// of the wave's queries see it; returns whether it holds codes that are no
// numbers, which it leaves out.  Weights are rounded to bf16 with their value's
// scale in them.
template <typename C, int DP, Cap CAP, bool EDGE>
__device__ __forceinline__ bool code_step(const AttnView& a, const char* k, const char* v, const char* pairs,
                                          const typename CodeTile<C, DP>::LaneAt& at,
                                          const uint4 (&q)[CodeTile<C, DP>::kQ], int j0, const Sight& row,
                                          Softmax& st, f32x16 (&acc)[DP / 32]) {
  using L = CodeTile<C, DP>;
  constexpr bool kI8 = std::is_same<C, code_i8>::value;
  constexpr int NB = DP / 32, kAhead = 2 * NB < 8 ? 2 * NB : 8;
  const bool odd = EDGE && L::any_odd(v);
  const uint32_t bits = EDGE ? lane_bits(row, j0) : 0;
  float mine = 1.f;
  if constexpr (!kI8) mine = key_scale(reinterpret_cast<const uint32_t*>(pairs)[threadIdx.x % 32]);
  f32x16 s[1] = {L::scores(k, at, q, mine)};
  uint32_t pair[16];
  lane_pairs(pairs, pair);
  if constexpr (kI8) {
#pragma unroll
    for (int x = 0; x < 16; ++x) s[0][x] *= key_scale(pair[x]);
  }
  if constexpr (CAP != Cap::none) cap_scores<CAP>(a, s);
  if constexpr (EDGE) mask_scores(s[0], bits);
  // the first pieces of the values come beside the softmax
  typename L::i32x2 vf[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) vf[i] = L::value_codes(v, at, i / NB, i % NB);
  __builtin_amdgcn_sched_barrier(0);
  softmax_step(CAP == Cap::none ? a.scale2 : 1.f, s, st, acc);
  bf16x8 p[2];
#pragma unroll
  for (int x = 0; x < 16; ++x) {
    float w = s[0][x] * value_scale(pair[x]);
    if (EDGE && !lane_sees(bits, x)) w = 0.f;  // not 0 times a NaN
    p[x / 8][x % 8] = static_cast<__bf16>(w);
  }
#pragma unroll
  for (int i = 0; i < 2 * NB; ++i) {
    const typename L::i32x2 c = vf[i % kAhead];
    bf16x8 x = code_numbers<C>(c[0], c[1]);
    if (EDGE && odd) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (!finite(static_cast<float>(x[e]))) x[e] = static_cast<__bf16>(0.f);
    }
    acc[i % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, p[i / NB], acc[i % NB], 0, 0, 0);
    if (i + kAhead < 2 * NB) vf[i % kAhead] = L::value_codes(v, at, (i + kAhead) / NB, (i + kAhead) % NB);
  }
  return odd;
}

}  // namespace kvx
