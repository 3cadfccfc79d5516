// attn_forward_kernels.h -- the attention kernels: chunks, single tokens and the
// join of their pieces.  S: what the cache holds (bf16_t, float, or a code of 8
// bits), A: AttnArgs, or AttnView for calls under a view.
#pragma once

#include "attn_few.h"
#include "attn_forward.h"
#include "attn_tile.h"
#include "attn_view_tile.h"

namespace kvx {
namespace {

// out row of query (row, head) from O^T registers and its sum; lane (n, h) has
// 4 columns of each 8.
template <typename T, int NB, typename Q>
__device__ __forceinline__ void store_out(const AttnArgs& a, const Q& q, int h,
                                          const f32x16 (&acc)[NB], const Softmax& st) {
  const int half = (threadIdx.x % 64) / 32;
  const float l = half_sum(st.l);
  const bool sees = sees_any(q);
  T* o = reinterpret_cast<T*>(a.out) + q.row * a.o_sr + (h * a.group + q.g) * a.o_sh;
#pragma unroll
  for (int db = 0; db < NB; ++db)
#pragma unroll
    for (int v = 0; v < 16; v += 4) {
      const int e = 32 * db + 2 * v + 4 * half;
      if (e >= a.d) continue;
      T x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = store_cvt<T>(sees ? acc[db][v + i] / l : 0.f);
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint2*>(o + e) = __builtin_bit_cast(uint2, x);
      else
        *reinterpret_cast<uint4*>(o + e) = __builtin_bit_cast(uint4, x);
    }
  if (a.lse && half == 0)
    a.lse[static_cast<int64_t>(q.row) * a.hq + h * a.group + q.g] =
        sees ? (st.m2 + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

// ---------------------------------------------------------------------------
// Chunks: S^T = K Q^T by 32 x 32 matrix instructions, so that a lane holds one
// query's scores and its weights are the second operand of O^T = V^T P^T as
// they stand: no weight changes lanes.  One pass with a running reference and
// sum.  Bound by the matrix units, and where heads are 256 wide by the LDS as
// much: each of 4 waves reads all of a tile's keys and values for 32 rows, about
// a thousand clocks, as its matrix work takes, and one wave a SIMD has to
// overlap the two.  Measured: 4096 tokens after 12k, heads 64 / 8 x 128: 1.85 ms,
// 1.04 PFLOP/s, where the card's power sets the clock (with zeros a fifth less
// time); 1531 tokens in 5627 slots, window 4096, heads 8 / 4 x 256, capped: 116 us,
// 445 TFLOP/s; fp32, 3 contexts of up to 257 in 1024 slots, heads 12 / 2 x 128:
// 56 us, 46 TFLOP/s of 154: a tile's scores, weights and products follow each
// other, its 232 workgroups do not divide the work evenly, and start and join
// take a quarter.
//
// 4 waves of 32 query rows share tiles of 64 slots (32 where rows have
// over 256 bytes), copied straight into LDS ahead of their use: values DEPTH
// tiles, keys one more.  One barrier per tile.  Depth 2 where one workgroup
// fills a compute unit, so that no other one hides the copies' latency, and
// LDS has room.  The scores of tile t + 1 are formed beside the weights of tile t,
// which need other units of the compute unit.
//
// Caches of 8 bits: codes are copied as they are, one tile ahead, and each wave
// turns a quarter of a tile into the rows of bf16 that the loops read, so that a
// number is converted once a workgroup.  Under a view a piece's start is found by
// every context's length (chunk_share).  Measured: 1021 tokens in 8192 slots of e4m3,
// heads 64 / 8 x 128: 314 us, 810 TFLOP/s; called without a pause, which lowers the
// clock, 375, of bf16 306: the conversion has no matrix work beside it but the other
// workgroup's (38% of clocks are matrix work, in bf16 56%).  Trees of 64 nodes, 8 contexts
// of up to 8k slots in int8, heads 28 / 4 x 128: 75 us (of bf16 64), 1.3 us a tile in
// bf16 and some 17 that do not depend on the tiles (start, first copies, masked
// tiles, 63 KB of instructions to fetch, the pieces' 64 KB); fp32, 3 contexts of up to 257 in
// 2900 slots, window 500 with sinks, heads 12 / 2 x 128: 45 us.
// ---------------------------------------------------------------------------

template <typename T, int DP>
constexpr int chunk_tile() { return DP * sizeof(T) <= 256 ? 64 : 32; }

// One turn of the chunk kernel's middle loop: the scores `next` of the tile
// whose keys are at k, the weights of the scores s, their products with the
// values at v, and next's largest scores.  A step is one LDS piece's matrix
// instructions and a share of the vector work, which the units do side by
// side; steps are kept apart, since the compiler left to itself read LDS just
// before each use and did the vector work in one go.  Pieces are read kAhead
// steps before their use.  Of the NS * 16 weights of a lane, three quarters
// come beside the scores, the last quarter beside the first half of the
// products (which do not need them), the largest scores beside the products.
template <typename T, int DP, Cap CAP, int NS>
__device__ __forceinline__ void middle_turn(const AttnArgs& a, const char* k, const char* v,
                                            const typename Tile<T, DP>::LaneAt& at,
                                            const uint4 (&q)[Tile<T, DP>::kQ], float c2,
                                            f32x16 (&s)[NS], f32x16 (&next)[NS], Softmax& st,
                                            f32x16 (&acc)[DP / 32], float& top) {
  using L = Tile<T, DP>;
  static_assert(L::kBf16, "");
  constexpr int KQ = L::kQ, kSteps = NS * KQ, kAheadK = 6, kAheadV = 4, NB = DP / 32;
  constexpr int kWeights = 16 * NS, kBeside = kWeights * 3 / 4, kLater = kWeights - kBeside;
  static_assert(2 * NS * NB == kSteps, "");
  uint4 kf[kAheadK + 1];
  bf16x8 vf[kAheadV + 1], b;
  // scores in log2 units less the reference: scale * s + shift.  Cap::part ones
  // are kept as the r of cap_part, which the line cap2 (1 - 2 r) brings there
  const float scale = CAP == Cap::part ? -2.f * a.cap2 : c2;
  const float shift = (CAP == Cap::part ? a.cap2 : 0.f) + (st.m2 == -INFINITY ? 0.f : -st.m2);
  float sum[2] = {0.f, 0.f};
  auto read_key = [&](int i) __attribute__((always_inline)) {
    kf[i % (kAheadK + 1)] = *reinterpret_cast<const uint4*>(
        k + i / KQ * 32 * L::kRowBytes + at.k[i % KQ % L::kKeyAt] + i % KQ / L::kKeyAt * L::kKeyAt * 32);
  };
  auto read_value = [&](int j) __attribute__((always_inline)) {
    vf[j % (kAheadV + 1)] = L::value_frag(v + j / (2 * NB) * 32 * L::kRowBytes, at, j / NB % 2, j % NB);
  };
  auto weigh = [&](int from, int to) __attribute__((always_inline)) {
#pragma unroll
    for (int e = from; e < to; ++e) {
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e / 16][e % 16], scale, shift));
      s[e / 16][e % 16] = p;
      sum[e % 2] += p;
    }
  };
#pragma unroll
  for (int i = 0; i < kAheadK; ++i) read_key(i);
#pragma unroll
  for (int u = 0; u < NS; ++u)
#pragma unroll
    for (int x = 0; x < 16; ++x) next[u][x] = 0.f;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    if (i + kAheadK < kSteps) read_key(i + kAheadK);
    if (i + kAheadV >= kSteps) read_value(i + kAheadV - kSteps);
    next[i / KQ] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
        __builtin_bit_cast(bf16x8, kf[i % (kAheadK + 1)]), __builtin_bit_cast(bf16x8, q[i % KQ]),
        next[i / KQ], 0, 0, 0);
    weigh(kBeside * i / kSteps, kBeside * (i + 1) / kSteps);
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    if (j + kAheadV < kSteps) read_value(j + kAheadV);
    if (j % NB == 0) {
      // weights rounded once to bf16 for the matrix instruction; the sum that
      // divides them keeps fp32
#pragma unroll
      for (int e = 0; e < 8; ++e) b[e] = static_cast<__bf16>(s[j / NB / 2][j / NB % 2 * 8 + e]);
    }
    acc[j % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[j % (kAheadV + 1)], b, acc[j % NB], 0, 0, 0);
    if (j < kSteps / 2) weigh(kBeside + 2 * kLater * j / kSteps, kBeside + 2 * kLater * (j + 1) / kSteps);
#pragma unroll
    for (int e = kWeights * j / kSteps; e < kWeights * (j + 1) / kSteps; ++e) {
      float x = next[e / 16][e % 16];
      if constexpr (CAP == Cap::part) next[e / 16][e % 16] = x = cap_part(a, x);
      if constexpr (CAP == Cap::tanh) next[e / 16][e % 16] = x = a.cap2 * cap_tanh(a, x);
      top = e == 0 ? x : CAP == Cap::part ? fminf(top, x) : fmaxf(top, x);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  top = CAP == Cap::part ? a.cap2 - 2.f * a.cap2 * -half_max(-top) : half_max(top) * c2;
  st.l += sum[0] + sum[1];
}

template <typename T, int DP>
constexpr int chunk_depth() { return DP * sizeof(T) == 512 ? 2 : 1; }

// Caches of 8 bits: a wave copies its share of a tile's codes into LDS a tile
// ahead, and turns it into bf16 rows when they have landed, once for all waves.
template <typename S, int DP, Cap CAP, typename A>
__global__ void __launch_bounds__(256, DP * sizeof(Numbers<S>) <= 256 ? 2 : 1)
    forward_chunk(A a, ForwardPlan fp) {
  using T = Numbers<S>;
  using L = Tile<T, DP>;
  constexpr bool kView = std::is_same<A, AttnView>::value, kCoded = sizeof(S) == 1;
  constexpr int TK = chunk_tile<T, DP>(), NS = TK / 32, NB = DP / 32;
  constexpr int kBytes = TK * L::kRowBytes;  // keys or values of a tile
  constexpr int kDepth = kCoded ? 1 : chunk_depth<T, DP>();
  // codes of 128 columns: two tiles of keys, so that two workgroups fit a unit
  constexpr int kKeys = kCoded && DP == 128 ? 2 : kDepth + 2, kValues = kDepth + 1;
  constexpr int kCopies = kBytes / 1024 / 4;  // of a wave, keys or values
  constexpr int kCodes = kCoded ? TK * DP : 0;  // bytes of a tile's keys or values as codes
  __shared__ __attribute__((aligned(16))) char lds[(kKeys + kValues) * kBytes + 2 * kCodes];
  const int lane = threadIdx.x % 64, n = lane % 32;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);

  ChunkShare sh;
  if constexpr (kView) {
    sh = chunk_share<TK>(a, fp.splits > 1);
    if (fp.splits > 1 && blockIdx.x == 0) {
      // strips that the caller's bounds allow for and that are not there
      const int none = fp.strips - sh.strips;
      for (int i = threadIdx.x; i < none * a.hkv; i += 256)
        fp.heads[i / none * fp.strips + sh.strips + i % none].pieces = 0;
    }
    if (__builtin_amdgcn_readfirstlane(sh.b) < 0) return;
  } else {
    // (head, piece, strip): consecutive units of an XCD share a head's cache;
    // later strips, which see more, first
    int id = xcd_remap(blockIdx.x, gridDim.x);
    sh.h = id / (fp.strips * fp.splits);
    id -= sh.h * fp.strips * fp.splits;
    sh.piece = id / fp.strips;
    sh.strip = fp.strips - 1 - id % fp.strips;

    // the strip's context: 64 contexts a step
    int b = -1, before = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
      int cnt = 0;
      if (b0 + lane < a.batch) {
        const Context c = context(a, b0 + lane);
        cnt = (c.m * a.group + kChunkRows - 1) / kChunkRows;
      }
      int sum = cnt;
#pragma unroll
      for (int i = 1; i < 64; i <<= 1) {
        const int y = __shfl_up(sum, i);
        if (lane >= i) sum += y;
      }
      const uint64_t past = __ballot(before + sum > sh.strip);
      if (past) {
        const int f = __ffsll(static_cast<unsigned long long>(past)) - 1;
        b = b0 + f;
        sh.qt = sh.strip - before - (__shfl(sum, f) - __shfl(cnt, f));
        break;
      }
      before += __shfl(sum, 63);
    }
    if (b < 0) {
      if (fp.splits > 1 && sh.piece == 0 && threadIdx.x == 0) fp.heads[sh.h * fp.strips + sh.strip].pieces = 0;
      return;
    }
    sh.b = b;
  }
  const int h = __builtin_amdgcn_readfirstlane(sh.h), b = __builtin_amdgcn_readfirstlane(sh.b);
  const int qt = __builtin_amdgcn_readfirstlane(sh.qt), strip = __builtin_amdgcn_readfirstlane(sh.strip);
  const int split = __builtin_amdgcn_readfirstlane(sh.piece);
  const int pieces = kView ? __builtin_amdgcn_readfirstlane(sh.pieces) : fp.splits;
  const int first = kView ? __builtin_amdgcn_readfirstlane(sh.first) : (h * fp.strips + strip) * fp.splits;
  const int step = kView ? __builtin_amdgcn_readfirstlane(sh.step) : 1;
  JoinHead* head = fp.heads + h * fp.strips + strip;
  const Context c = context(a, b);
  const int r0 = qt * kChunkRows, valid = min(kChunkRows, c.m * a.group - r0);
  const auto range = reach(a, c, r0, r0 + valid - 1);
  const typename LineOf<TK, A>::type line(range);
  const int per = (line.count + pieces - 1) / pieces;
  const int t0 = line.first + split * per, t1 = min(t0 + per, line.first + line.count);

  const auto qr = query_row(a, c, r0 + w * 32 + n);
  uint4 q[L::kQ];
  const T* qp = reinterpret_cast<const T*>(a.q) + qr.row * a.q_sr + (h * a.group + qr.g) * a.q_sh;
  L::load_q(q, w * 32 + n < valid ? qp : nullptr, a.d);
  // what the wave's rows see: together, and all of them
  const int rows_w = min(32, valid - w * 32);
  auto mine = range;
  if (rows_w > 0) {
    mine = reach(a, c, r0 + w * 32, r0 + w * 32 + rows_w - 1);
  } else {
    mine.lo = mine.hi = mine.alo = mine.ahi = 0;
    if constexpr (kView) mine.sink = mine.all_sink = 0;
  }

  f32x16 acc[NB];
  Softmax st;
#pragma unroll
  for (int db = 0; db < NB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;

  if (a.d < DP) {
    for (int i = threadIdx.x; i < static_cast<int>(sizeof(lds) / 16); i += 256)
      reinterpret_cast<uint4*>(lds)[i] = uint4{0, 0, 0, 0};
    __syncthreads();
  }
  const uint32_t l3 = lds_address(lds);
  const char* kb = a.c.k + h * a.c.sh * static_cast<int64_t>(sizeof(S));
  const char* vb = a.c.v + h * a.c.sh * static_cast<int64_t>(sizeof(S));
  Blocks<TK> kblocks, vblocks;
  bool odd = false;
  const typename L::LaneAt at = L::lane_at();
  // the queries are here: the compiler must not wait for them in the loop
  __builtin_amdgcn_s_waitcnt(0);
  // Codes: copy i of a wave takes R rows, a lane 16 codes of one, within 16 slots
  // that lie in one block; block numbers as forward_few's, one load for 64 of them.
  // The scales are of the tile whose keys, and of that whose values, were asked
  // for last.
  using R = CodeRows<DP>;
  constexpr int kCodeCopies = kCoded ? kCodes / 4096 : 1, kCodeStep = 4 * R::kRowsPerCopy;
  constexpr int kCodesAt = (kKeys + kValues) * kBytes, kSixteens = TK / 16;
  const int sub = lane / R::kChunks, code0 = lane % R::kChunks * 16;
  uint32_t kpair[kCodeCopies] = {}, vpair[kCodeCopies] = {};
  int base = t0, ids = 0;
  auto numbers = [&](int t) __attribute__((always_inline)) {
    if constexpr (kCoded) {
      const int j0 = min(line.slot(t + lane / kSixteens), (range.hi - 1) / TK * TK);
      return a.c.table[static_cast<int64_t>(b) * a.c.max_blocks + fdiv(a.c.bs, sixteen(range, j0 + 16 * (lane % kSixteens)))];
    }
    return 0;
  };
  // Runs of 16 slots bring some that the unit does not see, of which a fresh cache may
  // hold anything: as keys they are masked, and as values no reason to compute rows
  // again (1021 tokens in 8181 slots, heads 64 / 8 x 128, NaN behind them: 114 ms).  They
  // become zeros on their way, by their scale where codes are always numbers, by both
  // in e4m3; or, where that costs the loops registers and time, odd ones that the unit
  // sees are looked for in the end.  Measured (us; neither, zeros, looked for), heads 64 /
  // 8, int8, unless said otherwise: x 128 361, 357, 373; trees of 64 nodes 89, 89, 95; cap 50
  // 515, 504, 514; cap 1000 577, 640, 602 (e4m3 536, 593, 540); x 64 244, 254, 245.
  constexpr bool kZeros = DP > 64 && CAP != Cap::tanh;
  // where the last asked keys' rows begin, and so their values'
  int64_t code_at[kCodeCopies] = {};
  bool code_runs = false;
  auto copy_codes = [&](int t, const char* from, bool keys) __attribute__((always_inline)) {
    if constexpr (kCoded) {
      const bool table = a.c.table != nullptr;
      if (keys) {
        const int j0 = line.slot(t);
        const bool inside = range.inside(j0, TK);
        code_runs = a.c.run >= 16 && (table || inside || max(range.nearest(j0 + TK - 1) | 15, j0 + TK - 1) < a.c.capacity);
        if (code_runs && table && t - base >= 64 / kSixteens) {
          base = t;
          ids = numbers(t);
          __builtin_amdgcn_s_waitcnt(0);
        }
        const int64_t st = static_cast<uint32_t>(a.c.st);
        int64_t pair_at[kCodeCopies];
        if (inside && a.c.run >= TK) {
          const int32_t block = table ? __builtin_amdgcn_readlane(ids, (t - base) * kSixteens) : b;
          const int slot = (table ? j0 - fdiv(a.c.bs, j0) * static_cast<int>(a.c.bs.d) : j0) + w * R::kRowsPerCopy;
          const int64_t at = block * a.c.sb + slot * st, pair = block * a.scale.sb + slot * a.scale.st;
#pragma unroll
          for (int i = 0; i < kCodeCopies; ++i) {
            code_at[i] = at + i * kCodeStep * st;
            pair_at[i] = pair + (i * kCodeStep + sub) * a.scale.st;
          }
        } else {
#pragma unroll
          for (int i = 0; i < kCodeCopies; ++i) {
            const int row0 = i * kCodeStep + w * R::kRowsPerCopy;
            int j = range.nearest(j0 + row0 + sub);
            int32_t block = b;
            if (code_runs) {
              j = (inside ? j0 + (row0 & ~15) : sixteen(range, j0 + (row0 & ~15))) + row0 % 16;
              if (table) block = __builtin_amdgcn_readlane(ids, (t - base) * kSixteens + row0 / 16);
              const int slot = table ? j - fdiv(a.c.bs, j) * static_cast<int>(a.c.bs.d) : j;
              code_at[i] = block * a.c.sb + slot * st;
              j += sub;
            } else {
              block = cache_block(a.c, b, j);
              __builtin_amdgcn_s_waitcnt(0);
            }
            pair_at[i] = scale_offset(a.c, a.scale, block, j);
          }
        }
        // loaded here, not where paths part: where they meet the compiler would wait
#pragma unroll
        for (int i = 0; i < kCodeCopies; ++i) kpair[i] = a.scale.p[pair_at[i] + h * a.scale.sh];
      }
#pragma unroll
      for (int i = 0; i < kCodeCopies; ++i) {
        const uint32_t to = l3 + kCodesAt + (keys ? 0 : kCodes) + (i * 4 + w) * 1024;
        if (code_runs) {
          if (code0 < a.d) copy16(from + code_at[i], sub * static_cast<uint32_t>(a.c.st) + code0, to);
        } else {
          const int j = range.nearest(line.slot(t) + i * kCodeStep + w * R::kRowsPerCopy + sub);
          const char* at = from + cache_offset(a.c, cache_block(a.c, b, j), j) + code0;
          __builtin_amdgcn_s_waitcnt(0);
          if (code0 < a.d) copy16(at, to);
        }
        if (!keys) {
          vpair[i] = kpair[i];  // the same tile's, whose keys are here
          if constexpr (kZeros && std::is_same<S, code_i8>::value)
            if (!range.inside(line.slot(t), TK) &&
                range.misses(line.slot(t) + i * kCodeStep + w * R::kRowsPerCopy + sub, 1))
              vpair[i] = 0;
        }
      }
    }
  };
  auto copy_keys = [&](int t, int slot) __attribute__((always_inline)) {
    if constexpr (kCoded) {
      copy_codes(t, kb, true);
    } else {
      copy_tile<L, TK, 4, true, false>(a.c, kb, vb, b, line.slot(t), range, kblocks, a.d, w, l3 + slot * kBytes, 0);
      vblocks = kblocks;
      fetch_blocks(a.c, b, line.slot(t + 1), range.hi, kblocks);
    }
  };
  auto copy_values = [&](int t, int slot) __attribute__((always_inline)) {
    if constexpr (kCoded)
      copy_codes(t, vb, false);
    else
      copy_tile<L, TK, 4, false, true>(a.c, kb, vb, b, line.slot(t), range, vblocks, a.d, w, 0,
                                       l3 + (kKeys + slot) * kBytes);
  };
  // the wave's codes of tile t become rows of keys (or values) at `to`
  auto convert = [&](bool keys, int t, char* to) __attribute__((always_inline)) {
    if constexpr (kCoded) {
      const int j0 = line.slot(t);
      const bool edge = !keys && !range.inside(j0, TK);
#pragma unroll
      for (int i = 0; i < kCodeCopies; ++i) {
        uint4 x = *reinterpret_cast<const uint4*>(lds + kCodesAt + (keys ? 0 : kCodes) + (i * 4 + w) * 1024 + lane * 16);
        float f = keys ? key_scale(kpair[i]) : value_scale(vpair[i]);
        const int row = i * kCodeStep + w * R::kRowsPerCopy + lane / R::kChunks, chunk = 2 * (lane % R::kChunks);
        if constexpr (kZeros && std::is_same<S, code_e4m3>::value)
          if (edge && range.misses(j0 + row, 1)) {
            x = uint4{0, 0, 0, 0};
            f = 1.f;
          }
        const int swz = keys ? L::key_swz(row) : L::value_swz(row);
        *reinterpret_cast<bf16x8*>(to + row * L::kRowBytes + (chunk ^ swz) * 16) = code_numbers<S>(x.x, x.y, f);
        *reinterpret_cast<bf16x8*>(to + row * L::kRowBytes + ((chunk + 1) ^ swz) * 16) = code_numbers<S>(x.z, x.w, f);
      }
    }
  };
  if (t0 < t1) {
    if constexpr (kCoded) {
      if (a.c.table && a.c.run >= 16) ids = numbers(t0);
      __builtin_amdgcn_s_waitcnt(0);
    } else {
      fetch_blocks(a.c, b, line.slot(t0), range.hi, kblocks);
    }
    copy_keys(t0, 0);
    if constexpr (kCoded) {
      __builtin_amdgcn_s_waitcnt(0);
      convert(true, t0, lds);
    }
#pragma unroll
    for (int i = 0; i < kDepth; ++i) {
      if (t0 + i < t1) copy_values(t0 + i, i);
      if (t0 + i + 1 < t1) copy_keys(t0 + i + 1, i + 1);
    }
  }
  // Three loops, so that the one that matters has few registers to keep: tiles
  // before the first that all of the wave's queries see (windows), tiles that
  // all see, and the rest.  Where a score passes the reference by 2^kRoom in the
  // middle one, the sums are rescaled there; bf16 rows of 256 columns, short of
  // registers, leave it and enter it again with that tile's.  Measured (us, a
  // few calls in a row; there, left), scores of N(0, 1) and of ten times that: 4096 tokens in 16k, heads
  // 64 / 8 x 128: 1834, 1855 and 1872, 1929; fp32, 3 x 257 in 1024, heads 12 / 2 x
  // 128: 59, 58 and 60, 67; capped, 1531 in 5627, heads 8 / 4 x 256: 135, 127 and 138, 133.
  constexpr bool kInLoop = sizeof(T) == 4 || DP <= 128;
  const float c2 = CAP == Cap::none ? a.scale2 : 1.f;
  int kslot = 0, vslot = 0;  // of tile t
  auto after = [](int slot, int n, int by) { return slot + by >= n ? slot + by - n : slot + by; };
  // tiles that all waves' middle loops have, the first one and its turn apart
  int steady0 = 0, steady1 = 0;
  if constexpr (kCoded) {
    steady0 = max(t0, max(line.before, (range.alo + TK - 1) / TK - line.skip));
    steady1 = min(t1, line.until(range.ahi));
  }
  auto arrive = [&](int t) __attribute__((always_inline)) {
    // tile t's values and tile t + 1's keys have landed, those of kDepth - 1
    // more tiles may be in flight, and every wave is done with tile t - 1
    if constexpr (kCoded) {
      __builtin_amdgcn_s_waitcnt(0);  // the wave's codes and scales are here
      // Rows that are written have to be free: with three tiles of keys they are.
      // With two, those of tile t - 1 may still be read by waves that have just
      // entered a loop with it, or are at an edge; not by those that went on in
      // the middle one.
      if (kKeys == 2 && !(t - 1 > steady0 && t - 1 < steady1)) tile_barrier();
      if (t + 1 < t1) convert(true, t + 1, lds + after(kslot, kKeys, 1) * kBytes);
      convert(false, t, lds + (kKeys + vslot) * kBytes);
      if (t + 1 < t1) copy_values(t + 1, 0);
      if (t + 2 < t1) copy_keys(t + 2, 0);
      tile_barrier();
      __builtin_amdgcn_sched_barrier(0);
      return;
    }
    if (t + kDepth < t1)
      vm_wait<(kDepth - 1) * 2 * kCopies>();
    else
      vm_wait<0>();
    tile_barrier();
    if (t + kDepth < t1) copy_values(t + kDepth, after(vslot, kValues, kDepth));
    if (t + kDepth + 1 < t1) copy_keys(t + kDepth + 1, after(kslot, kKeys, kDepth + 1));
    __builtin_amdgcn_sched_barrier(0);
  };
  auto next_slots = [&]() __attribute__((always_inline)) {
    kslot = after(kslot, kKeys, 1);
    vslot = after(vslot, kValues, 1);
  };
  auto edges = [&](int t) __attribute__((always_inline)) {
    const int j0 = line.slot(t);
    if (mine.misses(j0, TK)) return;
    const char *k = lds + kslot * kBytes, *v = lds + (kKeys + vslot) * kBytes;
    // 32 slots at a time: the masks and checks want registers too
#pragma unroll 1
    for (int u = 0; u < NS; ++u) {
      const char *ku = k + u * 32 * L::kRowBytes, *vu = v + u * 32 * L::kRowBytes;
      if constexpr (kView)
        odd |= edge_step<T, DP, CAP>(a, ku, vu, at, q, j0 + 32 * u, qr.s, st, acc);
      else
        odd |= edge_step<T, DP, CAP>(a, ku, vu, at, q, j0 + 32 * u, qr.lo, qr.hi, st, acc);
    }
  };
  int t = t0;
  for (; t < t1 && line.slot(t) < mine.alo; ++t) {
    arrive(t);
    edges(t);
    next_slots();
  }
  const int tm = min(t1, line.until(mine.ahi));
  bool here = false;  // tile t has landed
  while (t < tm) {
    f32x16 s[NS];
    float top;
    auto score = [&](int slot, f32x16 (&s)[NS]) __attribute__((always_inline)) {
      const char* k = lds + slot * kBytes;
#pragma unroll
      for (int u = 0; u < NS; ++u) s[u] = L::scores(k + u * 32 * L::kRowBytes, at, q);
      if constexpr (CAP != Cap::part) {
        if constexpr (CAP == Cap::tanh) cap_scores<CAP>(a, s);
        top = top_score(c2, s);
      } else {
        f32x16 x[NS];
#pragma unroll
        for (int u = 0; u < NS; ++u)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            s[u][v] = cap_part(a, s[u][v]);
            x[u][v] = -s[u][v];
          }
        top = a.cap2 + top_score(2.f * a.cap2, x);
      }
    };
    if (!here) arrive(t);
    score(kslot, s);
    rescale(st, top, acc);
    while (true) {
      // the scores of tile t are within reach of the reference.  (After the
      // last tile the next one's are formed of what LDS holds, and not used.)
      f32x16 next[NS];
      const char *k = lds + after(kslot, kKeys, 1) * kBytes, *v = lds + (kKeys + vslot) * kBytes;
      if constexpr (L::kBf16) {
        middle_turn<T, DP, CAP, NS>(a, k, v, at, q, c2, s, next, st, acc, top);
      } else {
        score(after(kslot, kKeys, 1), next);
#pragma unroll
        for (int u = 0; u < NS; ++u) {
          weights(c2, s[u], st);
          L::template add_values<false>(v + u * 32 * L::kRowBytes, at, s[u], acc);
        }
      }
      next_slots();
      if (++t == tm) break;
      arrive(t);
      here = exceeds(st, top, kRoom);
      if (kInLoop) {
        if (here) rescale(st, top, acc);
        here = false;
      } else if (__builtin_expect(here, 0)) {
        break;
      }
#pragma unroll
      for (int u = 0; u < NS; ++u) s[u] = next[u];
    }
  }
  for (; t < t1; ++t) {
    arrive(t);
    edges(t);
    next_slots();
  }

  // a view's unit of one piece needs no join
  const bool whole = kView ? pieces == 1 : fp.splits == 1;
  float* part = fp.pieces + (static_cast<size_t>(first) + split * step) * piece_floats(kChunkRows, DP);
  if (fp.splits > 1 && split == 0 && threadIdx.x == 0) {
    int from, to;
    seeing(a, c, r0, from, to);
    *head = JoinHead{whole ? 0 : pieces, valid, c.q0, r0, h, first, from, to, b, step};
  }
  const int r = w * 32 + n;
  if (whole) {
    if (r < valid) store_out<T, NB>(a, qr, h, acc, st);
  } else {
    const float l = half_sum(st.l);
    if (r < valid) {
      if (lane < 32) reinterpret_cast<float2*>(part)[r] = float2{st.m2, l};
      float* o = part + 2 * kChunkRows + static_cast<size_t>(r) * DP;
#pragma unroll
      for (int db = 0; db < NB; ++db)
#pragma unroll
        for (int v = 0; v < 16; v += 4)
          *reinterpret_cast<float4*>(o + 32 * db + 2 * v + 4 * (lane / 32)) =
              float4{acc[db][v], acc[db][v + 1], acc[db][v + 2], acc[db][v + 3]};
    }
  }
  if (!odd) return;
  if constexpr (kCoded && !kZeros) {
    bool seen = false;
#pragma unroll 1
    for (int x = t0; x < t1 && !seen; ++x) {
      if ((line.slot(x) >= mine.alo && x < tm) || mine.misses(line.slot(x), TK)) continue;  // not at an edge
      seen = odd_codes<S>(a, b, h, range, line.slot(x), TK);
    }
    if (!seen) return;
  }
  vm_wait<0>();  // the rows that change are written again
#pragma unroll 1
  for (int r = 0; r < rows_w; ++r) {
    const auto u = query_row(a, c, r0 + w * 32 + r);
    float o[DP / 64];
    Softmax sm;
    const T* qu = reinterpret_cast<const T*>(a.q) + u.row * a.q_sr + (h * a.group + u.g) * a.q_sh;
    const auto slot = [&](int t) { return line.slot(t0 + t / NS) + t % NS * 32; };
    bool own;
    if constexpr (kView)
      own = careful_row<S, T, DP>(a, b, h, qu, u.s, (t1 - t0) * NS, slot, sm, o);
    else
      own = careful_row<T, DP>(a, b, h, qu, u.lo, u.hi, (t1 - t0) * NS, slot, sm, o);
    if (!own) continue;
    const int pr = w * 32 + r;
    if (!whole) {
      if (lane == 0) reinterpret_cast<float2*>(part)[pr] = float2{sm.m2, sm.l};
#pragma unroll
      for (int i = 0; i < DP / 64; ++i)
        part[2 * kChunkRows + static_cast<size_t>(pr) * DP + i * 64 + lane] = o[i];
    } else {
      T* to = reinterpret_cast<T*>(a.out) + u.row * a.o_sr + (h * a.group + u.g) * a.o_sh;
#pragma unroll
      for (int i = 0; i < DP / 64; ++i)
        if (i * 64 + lane < a.d) to[i * 64 + lane] = store_cvt<T>(o[i] / sm.l);
      if (a.lse && lane == 0)
        a.lse[static_cast<int64_t>(u.row) * a.hq + h * a.group + u.g] =
            (sm.m2 + __builtin_amdgcn_logf(sm.l)) * kLn2;
    }
  }
}

// ---------------------------------------------------------------------------
// Single tokens (and few): 32 query rows; the waves take different slots, each
// with its own ring of tiles in LDS and no barrier between them.  Bound by
// memory: every key and value is read once.  The (head, context, step) line of
// all work is cut into equal ranges, one a workgroup, so ragged contexts and
// single long ones fill the card alike; pieces of a unit are joined after.
// Measured, heads 28 / 4 x 128: 64 contexts of up to 8k slots, 605 MB in 118 us,
// 5.1 TB/s; one of 128k, 268 MB in 61 us, of which the join of 64 pieces takes 10;
// one of 300 slots, heads 12 / 2: 11.8 us, the latency of lengths, block
// numbers, two rounds of rows (two stages of copies are asked for one after the
// other) and two barriers.  Wider heads have fewer waves and stages, and registers
// that are read back from scratch memory once or twice a tile: heads 8 / 4, 64
// contexts of up to 8k slots: 256 columns 1208 MB in 357 us, 3.4 TB/s, 192 columns
// 906 MB in 381; fp32, 16 of up to 4k, 256 columns: 309 MB in 252.
// ---------------------------------------------------------------------------

template <typename S, int DP>
struct Decode {
  static constexpr bool kCoded = sizeof(S) == 1;
  // keys and values of 32 slots, and pairs of scales
  static constexpr int kStage = 2 * 32 * DP * sizeof(S) + (kCoded ? 128 : 0);
  static constexpr int kWaves = kCoded ? (DP == 256 ? 4 : 8) : ring_waves(kStage);
  static constexpr int kStages = kCoded ? (DP == 64 ? 4 : 2) : ring_stages(kStage);
  static constexpr int kStep = kWaves * 32;  // slots of a workgroup's step
  static_assert(kWaves * kStages * kStage <= 160 * 1024 && kStages * kStage >= 32 * DP * 4 + 256, "");
};

// Steps of a context's q tile: at least one, so that every row is written.
template <int STEP>
__device__ __forceinline__ int decode_steps(const AttnArgs& a, const Context& c, int qt) {
  int lo, hi;
  const int r0 = qt * kDecodeRows;
  seen_by(a, c, r0, min(r0 + kDecodeRows, c.m * a.group) - 1, lo, hi);
  lo &= ~31;
  return max(1, (hi - lo + STEP - 1) / STEP);
}
template <int STEP>
__device__ __forceinline__ int decode_steps(const AttnView& a, const Context& c, int qt) {
  const int r0 = qt * kDecodeRows;
  const ViewLine<32> line(reach(a, c, r0, min(r0 + kDecodeRows, c.m * a.group) - 1));
  return max(1, (line.count * 32 + STEP - 1) / STEP);
}

template <typename S, int DP, Cap CAP, typename A>
__global__ void __launch_bounds__((64 * Decode<S, DP>::kWaves), 1)
    forward_decode(A a, ForwardPlan fp) {
  using T = Numbers<S>;
  using L = typename TileOf<S, DP>::type;
  using D = Decode<S, DP>;
  constexpr bool kView = std::is_same<A, AttnView>::value, kCoded = D::kCoded;
  constexpr int NW = D::kWaves, NT = 64 * NW, NST = D::kStages, NB = DP / 32;
  constexpr int kBytes = 32 * L::kRowBytes;
  constexpr int kCopies = kBytes / 1024;
  __shared__ __attribute__((aligned(16))) char lds[NW * NST * D::kStage];
  const int tid = threadIdx.x, lane = tid % 64, n = lane % 32;
  const int w = __builtin_amdgcn_readfirstlane(tid / 64);
  JoinHead* head = fp.heads + blockIdx.x;

  // a unit is one step of the line where units are not split
  const bool whole = fp.splits == 1;
  const Share share = line_share(a, [&](int b) {
    const Context c = context(a, b);
    const int qts = (c.m * a.group + kDecodeRows - 1) / kDecodeRows;
    if (whole) return static_cast<int64_t>(qts);
    int64_t s = 0;
    for (int qt = 0; qt < qts; ++qt) s += decode_steps<D::kStep>(a, c, qt);
    return s;
  });
  if (tid == 0 && !whole) head->pieces = 0;
  const int64_t s0 = share.s0, s1 = share.s1, per = share.per;
  if (s0 >= s1) return;
  int h = share.h, b = share.b, step = share.step;
  Context c = context(a, b);
  int qt = whole ? step : 0;
  if (whole) step = 0;
  for (int x; step >= (x = decode_steps<D::kStep>(a, c, qt)); ++qt) step -= x;

  const typename L::LaneAt at = L::lane_at();
  const float c2 = CAP == Cap::none ? a.scale2 : 1.f;
  char* const ring = lds + w * NST * D::kStage;
  const uint32_t ring3 = lds_address(lds) + w * NST * D::kStage;

  for (int64_t s = s0; s < s1;) {
    // one unit: steps [step, step + cnt) of its `all`
    const int all = decode_steps<D::kStep>(a, c, qt);
    const int cnt = whole ? all : static_cast<int>(min<int64_t>(all - step, s1 - s));
    const int r0 = qt * kDecodeRows, valid = min(kDecodeRows, c.m * a.group - r0);
    const auto range = reach(a, c, r0, r0 + valid - 1);
    const int lo = range.lo, hi = range.hi;
    const typename LineOf<32, A>::type line(range);
    const int j_first = (lo & ~31) + (step * NW + w) * 32;
    // tiles of this wave: every NW-th of the range, as far as slots are seen
    int tiles = min(cnt, lo < hi && hi > j_first ? (hi - j_first + NW * 32 - 1) / (NW * 32) : 0);
    if constexpr (kView) tiles = min(cnt, max(line.count - (step * NW + w) + NW - 1, 0) / NW);
    const auto qr = query_row(a, c, r0 + n);
    uint4 q[L::kQ];
    const T* qp = reinterpret_cast<const T*>(a.q) + qr.row * a.q_sr + (h * a.group + qr.g) * a.q_sh;
    L::load_q(q, n < valid ? qp : nullptr, a.d);
    const char* kb = a.c.k + h * a.c.sh * static_cast<int64_t>(sizeof(S));
    const char* vb = a.c.v + h * a.c.sh * static_cast<int64_t>(sizeof(S));
    f32x16 acc[NB];
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;
    Softmax st;
    __syncthreads();  // LDS is free of the last unit's join
    if (a.d < DP) {
      // copies leave the chunks past head_dim alone: zeros
      for (int i = lane; i < NST * D::kStage / 16; i += 64)
        reinterpret_cast<uint4*>(ring)[i] = uint4{0, 0, 0, 0};
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }

    auto slot_of = [&](int t) __attribute__((always_inline)) {
      if constexpr (kView) return line.slot(step * NW + w + t * NW);
      return j_first + t * NW * 32;
    };
    Blocks<32> blocks;
    // block numbers are asked for where no wait for LDS follows soon: such a
    // wait covers scalar loads too
    auto copy = [&](int t) __attribute__((always_inline)) {
      const int j0 = slot_of(t);
      const uint32_t to = ring3 + t % NST * D::kStage;
      copy_tile<L, 32, 1, true, true>(a.c, kb, vb, b, j0, range, blocks, a.d, 0, to, to + kBytes);
      if constexpr (kCoded) {
        const int j = range.nearest(j0 + n);
        int32_t block = b;
        if (a.c.table) {
          if (a.c.run >= 16 && range.inside(j0, 32))
            block = n < 16 ? blocks.id[0] : blocks.id[1];
          else
            block = cache_block(a.c, b, j);
        }
        if (lane < 32)
          copy4(reinterpret_cast<const char*>(a.scale.p + scale_offset(a.c, a.scale, block, j) + h * a.scale.sh),
                to + 2 * kBytes);
      }
    };
    constexpr int kFlight = 2 * kCopies + (kCoded ? 1 : 0);  // copies of a tile
    bool odd = false;
    if (tiles > 0) fetch_blocks(a.c, b, slot_of(0), hi, blocks);
    for (int t = 0; t < NST - 1 && t < tiles; ++t) {
      copy(t);
      fetch_blocks(a.c, b, slot_of(t + 1), hi, blocks);
    }
    // the queries are here: the compiler must not wait for them in the loop
    __builtin_amdgcn_s_waitcnt(0);
    for (int t = 0; t < tiles; ++t) {
      // the stage that tile t + NST - 1 takes was read a tile ago, its values
      // used before this line
      __builtin_amdgcn_sched_barrier(0);
      if (t + NST - 1 < tiles) {
        copy(t + NST - 1);
        // all but the last NST - 1 tiles' copies have landed
        vm_wait<(NST - 1) * kFlight>();
      } else {
        vm_wait<0>();
      }
      const char* k = ring + t % NST * D::kStage;
      const char* v = k + kBytes;
      const int j0 = slot_of(t);
      if constexpr (kCoded) {
        if (range.all_see(j0, 32))
          code_step<S, DP, CAP, false>(a, k, v, v + kBytes, at, q, j0, qr.s, st, acc);
        else
          odd |= code_step<S, DP, CAP, true>(a, k, v, v + kBytes, at, q, j0, qr.s, st, acc);
      } else if (range.all_see(j0, 32)) {
        f32x16 sc[1] = {L::scores(k, at, q)};
        if constexpr (CAP != Cap::none) cap_scores<CAP>(a, sc);
        if constexpr (L::kBf16) {
          // the first pieces of the values come beside the softmax
          constexpr int kAhead = 2 * NB < 8 ? 2 * NB : 8;
          bf16x8 vf[kAhead];
#pragma unroll
          for (int i = 0; i < kAhead; ++i) vf[i] = L::value_frag(v, at, i / NB, i % NB);
          __builtin_amdgcn_sched_barrier(0);
          softmax_step(c2, sc, st, acc);
          bf16x8 p[2];
#pragma unroll
          for (int e = 0; e < 16; ++e) p[e / 8][e % 8] = static_cast<__bf16>(sc[0][e]);
#pragma unroll
          for (int i = 0; i < 2 * NB; ++i) {
            acc[i % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i % kAhead], p[i / NB], acc[i % NB], 0, 0, 0);
            if (i + kAhead < 2 * NB) vf[i % kAhead] = L::value_frag(v, at, (i + kAhead) / NB, (i + kAhead) % NB);
          }
        } else {
          softmax_step(c2, sc, st, acc);
          L::template add_values<false>(v, at, sc[0], acc);
        }
      } else if constexpr (kView) {
        odd |= edge_step<T, DP, CAP>(a, k, v, at, q, j0, qr.s, st, acc);
      } else {
        odd |= edge_step<T, DP, CAP>(a, k, v, at, q, j0, qr.lo, qr.hi, st, acc);
      }
      __builtin_amdgcn_sched_barrier(0);
      fetch_blocks(a.c, b, slot_of(t + NST), hi, blocks);
    }

    // the waves' results through LDS: each in its own ring, rows of DP floats,
    // 16-byte pieces swizzled by the row; then (m2, l)
    const float l = half_sum(st.l);
    if (n < valid) {
      float4* o = reinterpret_cast<float4*>(ring) + n * (DP / 4);
#pragma unroll
      for (int db = 0; db < NB; ++db)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          o[(8 * db + 2 * x + lane / 32) ^ (n & 7)] =
              float4{acc[db][4 * x], acc[db][4 * x + 1], acc[db][4 * x + 2], acc[db][4 * x + 3]};
      if (lane < 32)
        reinterpret_cast<float2*>(ring + 32 * DP * 4)[n] = float2{st.m2, l};
    }
    if (odd) {
#pragma unroll 1
      for (int r = 0; r < valid; ++r) {
        const auto u = query_row(a, c, r0 + r);
        float o[DP / 64];
        Softmax sm;
        const T* qu = reinterpret_cast<const T*>(a.q) + u.row * a.q_sr + (h * a.group + u.g) * a.q_sh;
        bool own;
        if constexpr (kView)
          own = careful_row<S, T, DP>(a, b, h, qu, u.s, tiles, slot_of, sm, o);
        else
          own = careful_row<T, DP>(a, b, h, qu, u.lo, u.hi, tiles, slot_of, sm, o);
        if (!own) continue;
#pragma unroll
        for (int i = 0; i < DP / 64; ++i) {
          const int e = i * 64 + lane;
          reinterpret_cast<float*>(ring)[r * DP + ((e / 4) ^ (r & 7)) * 4 + e % 4] = o[i];
        }
        if (lane == 0) reinterpret_cast<float2*>(ring + 32 * DP * 4)[r] = float2{sm.m2, sm.l};
      }
    }
    __syncthreads();
    const bool begins = step == 0, ends = step + cnt == all;
    float* part = fp.pieces + (2 * static_cast<size_t>(blockIdx.x) + (begins ? 1 : 0)) * piece_floats(kDecodeRows, DP);
    for (int i = tid; i < valid * (DP / 4); i += NT) {
      const int r = i / (DP / 4), e = i % (DP / 4);
      float2 ml[NW];
      float m2 = -INFINITY;
#pragma unroll
      for (int x = 0; x < NW; ++x) {
        ml[x] = reinterpret_cast<const float2*>(lds + x * NST * D::kStage + 32 * DP * 4)[r];
        m2 = fmaxf(m2, ml[x].x);
      }
      float lsum = 0.f;
      float4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < NW; ++x) {
        const float f = ml[x].x == m2 ? 1.f : __builtin_amdgcn_exp2f(ml[x].x - m2);
        const float4 y = reinterpret_cast<const float4*>(lds + x * NST * D::kStage)[r * (DP / 4) + (e ^ (r & 7))];
        lsum += f * ml[x].y;
        o.x += f * y.x;
        o.y += f * y.y;
        o.z += f * y.z;
        o.w += f * y.w;
      }
      if (begins && ends) {
        const auto u = query_row(a, c, r0 + r);
        const bool sees = sees_any(u);
        if (4 * e < a.d) {
          T* to = reinterpret_cast<T*>(a.out) + u.row * a.o_sr + (h * a.group + u.g) * a.o_sh + 4 * e;
          const float x[4] = {o.x, o.y, o.z, o.w};
          T y[4];
#pragma unroll
          for (int z = 0; z < 4; ++z) y[z] = store_cvt<T>(sees ? x[z] / lsum : 0.f);
          if constexpr (sizeof(T) == 2)
            *reinterpret_cast<uint2*>(to) = __builtin_bit_cast(uint2, y);
          else
            *reinterpret_cast<uint4*>(to) = __builtin_bit_cast(uint4, y);
        }
        if (a.lse && e == 0)
          a.lse[static_cast<int64_t>(u.row) * a.hq + h * a.group + u.g] =
              sees ? (m2 + __builtin_amdgcn_logf(lsum)) * kLn2 : -INFINITY;
      } else {
        reinterpret_cast<float4*>(part + 2 * kDecodeRows)[i] = o;
        if (e == 0) reinterpret_cast<float2*>(part)[r] = float2{m2, lsum};
      }
    }
    if (begins && !ends && tid == 0) {
      // the unit's other pieces are the first ones of the next workgroups
      const int64_t end = s - step + all;
      int from, to;
      seeing(a, c, r0, from, to);
      *head = JoinHead{static_cast<int32_t>((end - 1) / per - blockIdx.x + 1), valid, c.q0, r0, h,
                       static_cast<int32_t>(2 * blockIdx.x + 1), from, to, b};
    }
    s += whole ? 1 : cnt;
    step = 0;
    if (s < s1) {
      // the next q tile, of this context or one with new tokens after it
      ++qt;
      while (qt * kDecodeRows >= c.m * a.group) {
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

// Joins the pieces of units: W waves a query row, wave w the pieces w, w + W,
// .., whose sums are then added in the waves' order.  Four for single tokens,
// whose few rows have many pieces; one for chunks.  Bound by latency for single
// tokens (28 rows of 64 pieces: 10 us) and by the pieces' reading for chunks (96
// strips of 5 pieces x 256 columns, 63 MB: 15.5 us; trees of 64 nodes, heads 28 x 128,
// 8 contexts in 256 pieces, 17 MB: 11.5, most of it the wait for what a row's pieces
// and its context are).
template <typename T, int DP, int W, typename A>
__global__ void __launch_bounds__(256) forward_join(A a, ForwardPlan fp) {
  constexpr int PER = DP / 64;
  __shared__ float sums[4][DP];
  __shared__ float part_l[4];
  const JoinHead hd = fp.heads[blockIdx.x];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, w = wave % W;
  if (hd.pieces == 0) return;
  const int unit_rows = fp.decode ? kDecodeRows : kChunkRows;
  const size_t size = piece_floats(unit_rows, DP);
  // decode: piece 0 is slot 1 of its workgroup, the others slot 0 of the next ones
  auto piece = [&](int p) __attribute__((always_inline)) {
    const size_t at = fp.decode ? (p == 0 ? hd.first : hd.first - 1 + 2 * static_cast<size_t>(p)) : hd.first + static_cast<size_t>(p) * hd.step;
    return fp.pieces + at * size;
  };
  // the grid has the rows that the caller's bound on new tokens gives
  for (int r0 = blockIdx.y * (4 / W); r0 < hd.rows; r0 += gridDim.y * (4 / W)) {
    const int r = r0 + wave / W;
    const int rc = min(r, hd.rows - 1);  // rows past the last one are not stored
    float m2 = -INFINITY;
    for (int p = lane; p < hd.pieces; p += 64) m2 = fmaxf(m2, reinterpret_cast<const float2*>(piece(p))[rc].x);
#pragma unroll
    for (int i = 32; i; i >>= 1) m2 = fmaxf(m2, __shfl_xor(m2, i));
    float l = 0.f, o[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) o[i] = 0.f;
#pragma unroll 8
    for (int p = w; p < hd.pieces; p += W) {
      const float* part = piece(p);
      const float2 ml = reinterpret_cast<const float2*>(part)[rc];
      const float* x = part + 2 * unit_rows + static_cast<size_t>(rc) * DP + lane * PER;
      const float f = ml.x == m2 ? 1.f : __builtin_amdgcn_exp2f(ml.x - m2);
      l += f * ml.y;
#pragma unroll
      for (int i = 0; i < PER; ++i) o[i] += f * x[i];
    }
    if constexpr (W > 1) {
      static_assert(W == 4, "the waves of a workgroup");
#pragma unroll
      for (int i = 0; i < PER; ++i) sums[w][lane * PER + i] = o[i];
      if (lane == 0) part_l[w] = l;
      __syncthreads();
      l = (part_l[0] + part_l[1]) + (part_l[2] + part_l[3]);
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int e = lane * PER + i;
        o[i] = (sums[0][e] + sums[1][e]) + (sums[2][e] + sums[3][e]);
      }
      __syncthreads();
    }
    if (r >= hd.rows || w > 0) continue;
    const int rr = hd.g0 + r, tok = fdiv(a.by_group, rr), g = rr - tok * a.group;
    const int64_t row = hd.row0 + tok;
    const int head = hd.h * a.group + g;
    bool sees = r >= hd.from && r < hd.to;
    if constexpr (std::is_same<A, AttnView>::value) sees = sees_any(sight(a, context(a, hd.b), tok));
    T* to = reinterpret_cast<T*>(a.out) + row * a.o_sr + head * a.o_sh;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (lane * PER + i < a.d) to[lane * PER + i] = store_cvt<T>(sees ? o[i] / l : 0.f);
    if (a.lse && lane == 0) a.lse[row * a.hq + head] = sees ? (m2 + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
  }
}

// Joins the pieces of units of few query rows.  SPREAD: units of hundreds of
// pieces (few long contexts), a workgroup of 16 waves a row, which ask for all at
// once and whose sums are added in the waves' order: 28 rows of 128 pieces 7.4
// us, by 4 waves 15.8.  Otherwise a wave a row: 448 units of 7 rows 5.9 us.
template <typename T, int DP, bool SPREAD>
__global__ void __launch_bounds__(SPREAD ? 1024 : 256) few_join(AttnView a, ForwardPlan fp) {
  constexpr int PER = DP / 64, W = SPREAD ? 16 : 1;
  __shared__ float sums[W][DP];
  __shared__ float part_l[W];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, w = SPREAD ? wave : 0;
  const size_t size = piece_floats(kFewRows, DP);
  // a workgroup's heads
  const int share = (fp.grid + gridDim.x - 1) / gridDim.x, end = min<int>(fp.grid, (blockIdx.x + 1) * share);
  for (int x0 = blockIdx.x * share; x0 < end; x0 += 64) {
    uint64_t todo = __ballot(x0 + lane < end && fp.heads[min(x0 + lane, end - 1)].pieces > 0);
    for (; todo; todo &= todo - 1) {
      const JoinHead hd = fp.heads[x0 + __ffsll(static_cast<unsigned long long>(todo)) - 1];
      auto piece = [&](int p) __attribute__((always_inline)) {
        return fp.pieces + (p == 0 ? hd.first : hd.first - 1 + 2 * static_cast<size_t>(p)) * size;
      };
      const int rows = SPREAD ? 1 : 4;  // of a workgroup's turn
      for (int r = blockIdx.y * rows + (SPREAD ? 0 : wave); r < hd.rows; r += gridDim.y * rows) {
        const int tok = fdiv(a.by_group, hd.g0 + r), g = hd.g0 + r - tok * a.group;
        const bool sees = sees_any(sight(a, context(a, hd.b), tok));
        const int64_t row = hd.row0 + tok;
        const int head = hd.h * a.group + g;
        float m2 = -INFINITY;
        for (int p = lane; p < hd.pieces; p += 64)
          m2 = fmaxf(m2, reinterpret_cast<const float2*>(piece(p))[r].x);
#pragma unroll
        for (int i = 32; i; i >>= 1) m2 = fmaxf(m2, __shfl_xor(m2, i));
        float l = 0.f, o[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) o[i] = 0.f;
#pragma unroll 8
        for (int p = w; p < hd.pieces; p += W) {
          const float* part = piece(p);
          const float2 ml = reinterpret_cast<const float2*>(part)[r];
          const float* x = part + 2 * kFewRows + static_cast<size_t>(r) * DP + lane * PER;
          const float f = ml.x == m2 ? 1.f : __builtin_amdgcn_exp2f(ml.x - m2);
          l += f * ml.y;
#pragma unroll
          for (int i = 0; i < PER; ++i) o[i] += f * x[i];
        }
        T* to = reinterpret_cast<T*>(a.out) + row * a.o_sr + head * a.o_sh;
        if constexpr (SPREAD) {
#pragma unroll
          for (int i = 0; i < PER; ++i) sums[w][lane * PER + i] = o[i];
          if (lane == 0) part_l[w] = l;
          __syncthreads();
          const int e = threadIdx.x, used = min(hd.pieces, W);
          if (e < a.d) {
            float x = 0.f;
            l = 0.f;
            for (int i = 0; i < used; ++i) {
              x += sums[i][e];
              l += part_l[i];
            }
            to[e] = store_cvt<T>(sees ? x / l : 0.f);
          }
          __syncthreads();
        } else {
#pragma unroll
          for (int i = 0; i < PER; ++i)
            if (lane * PER + i < a.d) to[lane * PER + i] = store_cvt<T>(sees ? o[i] / l : 0.f);
        }
        if (a.lse && lane == 0 && w == 0)
          a.lse[row * a.hq + head] = sees ? (m2 + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
      }
    }
  }
}

// Launches the kernels of one call.
template <typename S, int DP, typename A>
hipError_t run_attention(const A& a, const ForwardPlan& p, hipStream_t st) {
  using T = Numbers<S>;
  constexpr Cap kPart = sizeof(T) == 2 ? Cap::part : Cap::tanh;
  const bool cap = a.cap2 != 0.f, part = a.cap2 <= static_cast<float>(kPartCap * kLog2e);
  auto* kernel = p.decode ? !cap   ? forward_decode<S, DP, Cap::none, A>
                            : part ? forward_decode<S, DP, kPart, A>
                                   : forward_decode<S, DP, Cap::tanh, A>
                 : !cap   ? forward_chunk<S, DP, Cap::none, A>
                 : part   ? forward_chunk<S, DP, kPart, A>
                          : forward_chunk<S, DP, Cap::tanh, A>;
  dim3 block(p.decode ? 64 * Decode<S, DP>::kWaves : 256);
  if constexpr (std::is_same<A, AttnView>::value && sizeof(S) <= 2) {
    if (p.few) {
      kernel = !cap   ? forward_few<S, DP, Cap::none>
               : part ? forward_few<S, DP, Cap::part>
                      : forward_few<S, DP, Cap::tanh>;
      block = dim3(64 * Few<S, DP>::kWaves);
    }
  }
  const hipError_t e = launch_on(kernel, dim3(p.grid), block, st, a, p);
  if (p.splits == 1) return e;
  if (e != hipSuccess) return e;
  if constexpr (std::is_same<A, AttnView>::value && sizeof(S) <= 2)
    if (p.few)
      return int64_t(a.batch) * a.hkv <= 32
                 ? launch_on(few_join<T, DP, true>, dim3(32, p.join_rows), dim3(1024), st, a, p)
                 : launch_on(few_join<T, DP, false>, dim3(p.grid, (p.join_rows + 3) / 4), dim3(256), st, a, p);
  return p.decode
             ? launch_on(forward_join<T, DP, 4, A>, dim3(p.grid, p.join_rows), dim3(256), st, a, p)
             : launch_on(forward_join<T, DP, 1, A>, dim3(p.strips * a.hkv, p.join_rows / 4), dim3(256), st, a, p);
}

}  // namespace
}  // namespace kvx
