// attn_forward_d.hip -- the attention kernels of one padded head_dim
// (KVX_ATTN_DP = 64, 128 or 256), both dtypes.
#include "attn_forward.h"
#include "attn_tile.h"

namespace kvx {
namespace {

// out row of query (row, head) from O^T registers and its sum; lane (n, h) has
// 4 columns of each 8.
template <typename T, int NB>
__device__ __forceinline__ void store_out(const AttnArgs& a, const QueryRow& q, int h,
                                          const f32x16 (&acc)[NB], const Softmax& st) {
  const int half = (threadIdx.x % 64) / 32;
  const float l = half_sum(st.l);
  const bool sees = q.lo < q.hi;
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
// overlap the two.  Measured: 4096 tokens after 12k, heads 64 / 8 x 128: 1.88 ms,
// 1.02 PFLOP/s, where the card's power sets the clock (with zeros a fifth less
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

template <typename T, int DP, Cap CAP>
__global__ void __launch_bounds__(256, DP * sizeof(T) <= 256 ? 2 : 1)
    forward_chunk(AttnArgs a, ForwardPlan fp) {
  using L = Tile<T, DP>;
  constexpr int TK = chunk_tile<T, DP>(), NS = TK / 32, NB = DP / 32;
  constexpr int kBytes = TK * L::kRowBytes;  // keys or values of a tile
  constexpr int kDepth = chunk_depth<T, DP>(), kKeys = kDepth + 2, kValues = kDepth + 1;
  constexpr int kCopies = kBytes / 1024 / 4;  // of a wave, keys or values
  __shared__ __attribute__((aligned(16))) char lds[(kKeys + kValues) * kBytes];
  const int lane = threadIdx.x % 64, n = lane % 32;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);

  // (head, piece, strip): consecutive units of an XCD share a head's cache;
  // later strips, which see more, first
  int id = xcd_remap(blockIdx.x, gridDim.x);
  const int h = id / (fp.strips * fp.splits);
  id -= h * fp.strips * fp.splits;
  const int split = id / fp.strips, strip = fp.strips - 1 - id % fp.strips;

  // the strip's context: 64 contexts a step
  int b = -1, qt = 0, before = 0;
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
    const uint64_t past = __ballot(before + sum > strip);
    if (past) {
      const int f = __ffsll(static_cast<unsigned long long>(past)) - 1;
      b = b0 + f;
      qt = strip - before - (__shfl(sum, f) - __shfl(cnt, f));
      break;
    }
    before += __shfl(sum, 63);
  }
  JoinHead* head = fp.heads + h * fp.strips + strip;
  if (b < 0) {
    if (fp.splits > 1 && split == 0 && threadIdx.x == 0) head->pieces = 0;
    return;
  }
  b = __builtin_amdgcn_readfirstlane(b);
  qt = __builtin_amdgcn_readfirstlane(qt);
  const Context c = context(a, b);
  const int r0 = qt * kChunkRows, valid = min(kChunkRows, c.m * a.group - r0);
  int lo, hi;
  seen_by(a, c, r0, r0 + valid - 1, lo, hi);
  const int tiles = lo < hi ? (hi + TK - 1) / TK - lo / TK : 0;
  const int per = (tiles + fp.splits - 1) / fp.splits;
  const int t0 = lo / TK + split * per, t1 = min(t0 + per, lo / TK + tiles);

  const QueryRow qr = query_row(a, c, r0 + w * 32 + n);
  uint4 q[L::kQ];
  const T* qp = reinterpret_cast<const T*>(a.q) + qr.row * a.q_sr + (h * a.group + qr.g) * a.q_sh;
  L::load_q(q, w * 32 + n < valid ? qp : nullptr, a.d);
  // what the wave's rows see: together, and all of them
  const int rows_w = min(32, valid - w * 32);
  int wlo = 0, whi = 0, alo = 0, ahi = 0;
  if (rows_w > 0) {
    const int rw = r0 + w * 32;
    seen_by(a, c, rw, rw + rows_w - 1, wlo, whi);
    seen_by(a, c, rw, rw, alo, ahi);
    seen_by(a, c, rw + rows_w - 1, rw + rows_w - 1, alo, whi);
  }

  f32x16 acc[NB];
  Softmax st;
#pragma unroll
  for (int db = 0; db < NB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;

  if (a.d < DP) {
    for (int i = threadIdx.x; i < (kKeys + kValues) * kBytes / 16; i += 256)
      reinterpret_cast<uint4*>(lds)[i] = uint4{0, 0, 0, 0};
    __syncthreads();
  }
  const uint32_t l3 = lds_address(lds);
  const char* kb = a.c.k + h * a.c.sh * static_cast<int64_t>(sizeof(T));
  const char* vb = a.c.v + h * a.c.sh * static_cast<int64_t>(sizeof(T));
  Blocks<TK> kblocks, vblocks;
  bool odd = false;
  const typename L::LaneAt at = L::lane_at();
  // the queries are here: the compiler must not wait for them in the loop
  __builtin_amdgcn_s_waitcnt(0);
  auto copy_keys = [&](int t, int slot) __attribute__((always_inline)) {
    copy_tile<T, DP, TK, 4, true, false>(a.c, kb, vb, b, t * TK, lo, hi, kblocks, a.d, w,
                                         l3 + slot * kBytes, 0);
    vblocks = kblocks;
    fetch_blocks(a.c, b, t * TK + TK, hi, kblocks);
  };
  auto copy_values = [&](int t, int slot) __attribute__((always_inline)) {
    copy_tile<T, DP, TK, 4, false, true>(a.c, kb, vb, b, t * TK, lo, hi, vblocks, a.d, w, 0,
                                         l3 + (kKeys + slot) * kBytes);
  };
  if (t0 < t1) {
    fetch_blocks(a.c, b, t0 * TK, hi, kblocks);
    copy_keys(t0, 0);
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
  auto arrive = [&](int t) __attribute__((always_inline)) {
    // tile t's values and tile t + 1's keys have landed, those of kDepth - 1
    // more tiles may be in flight, and every wave is done with tile t - 1
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
    if (t * TK >= whi || t * TK + TK <= wlo) return;
    const char *k = lds + kslot * kBytes, *v = lds + (kKeys + vslot) * kBytes;
    // 32 slots at a time: the masks and checks want registers too
#pragma unroll 1
    for (int u = 0; u < NS; ++u)
      odd |= edge_step<T, DP, CAP>(a, k + u * 32 * L::kRowBytes, v + u * 32 * L::kRowBytes, at, q,
                                   t * TK + 32 * u, qr.lo, qr.hi, st, acc);
  };
  int t = t0;
  for (; t < t1 && t * TK < alo; ++t) {
    arrive(t);
    edges(t);
    next_slots();
  }
  const int tm = min(t1, ahi / TK);
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

  const int unit = h * fp.strips + strip;
  float* part = fp.pieces + (static_cast<size_t>(unit) * fp.splits + split) * piece_floats(kChunkRows, DP);
  if (fp.splits > 1 && split == 0 && threadIdx.x == 0) {
    int from, to;
    seeing(a, c, r0, from, to);
    *head = JoinHead{fp.splits, valid, c.q0, r0, h, unit * fp.splits, from, to};
  }
  const int r = w * 32 + n;
  if (fp.splits == 1) {
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
  vm_wait<0>();  // the rows that change are written again
#pragma unroll 1
  for (int r = 0; r < rows_w; ++r) {
    const QueryRow u = query_row(a, c, r0 + w * 32 + r);
    float o[DP / 64];
    Softmax sm;
    if (!careful_row<T, DP>(
            a, b, h, reinterpret_cast<const T*>(a.q) + u.row * a.q_sr + (h * a.group + u.g) * a.q_sh,
            u.lo, u.hi, (t1 - t0) * NS, [&](int t) { return t0 * TK + t * 32; }, sm, o))
      continue;
    const int pr = w * 32 + r;
    if (fp.splits > 1) {
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

template <typename T, int DP>
struct Decode {
  static constexpr int kStage = 2 * 32 * DP * sizeof(T);  // keys and values of 32 slots
  static constexpr int kWaves = ring_waves(kStage);
  static constexpr int kStages = ring_stages(kStage);
  static constexpr int kStep = kWaves * 32;  // slots of a workgroup's step
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

template <typename T, int DP, Cap CAP>
__global__ void __launch_bounds__((64 * Decode<T, DP>::kWaves), 1)
    forward_decode(AttnArgs a, ForwardPlan fp) {
  using L = Tile<T, DP>;
  using D = Decode<T, DP>;
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
    int lo, hi, alo, ahi, xlo, xhi;
    seen_by(a, c, r0, r0 + valid - 1, lo, hi);
    seen_by(a, c, r0, r0, xlo, ahi);                          // the least that any row's end is
    seen_by(a, c, r0 + valid - 1, r0 + valid - 1, alo, xhi);  // the most that any row's start is
    const int j_first = (lo & ~31) + (step * NW + w) * 32;
    // tiles of this wave: every NW-th of the range, as far as slots are seen
    const int tiles = min(cnt, lo < hi && hi > j_first ? (hi - j_first + NW * 32 - 1) / (NW * 32) : 0);
    const QueryRow qr = query_row(a, c, r0 + n);
    uint4 q[L::kQ];
    const T* qp = reinterpret_cast<const T*>(a.q) + qr.row * a.q_sr + (h * a.group + qr.g) * a.q_sh;
    L::load_q(q, n < valid ? qp : nullptr, a.d);
    const char* kb = a.c.k + h * a.c.sh * static_cast<int64_t>(sizeof(T));
    const char* vb = a.c.v + h * a.c.sh * static_cast<int64_t>(sizeof(T));
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

    auto slot_of = [&](int t) __attribute__((always_inline)) { return j_first + t * NW * 32; };
    Blocks<32> blocks;
    // block numbers are asked for where no wait for LDS follows soon: such a
    // wait covers scalar loads too
    auto copy = [&](int t) __attribute__((always_inline)) {
      copy_tile<T, DP, 32, 1>(a.c, kb, vb, b, slot_of(t), lo, hi, blocks, a.d, 0,
                              ring3 + t % NST * D::kStage, ring3 + t % NST * D::kStage + kBytes);
    };
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
        vm_wait<(NST - 1) * 2 * kCopies>();
      } else {
        vm_wait<0>();
      }
      const char* k = ring + t % NST * D::kStage;
      const char* v = k + kBytes;
      const int j0 = slot_of(t);
      if (j0 >= alo && j0 + 32 <= ahi) {
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
        const QueryRow u = query_row(a, c, r0 + r);
        float o[DP / 64];
        Softmax sm;
        if (!careful_row<T, DP>(
                a, b, h, reinterpret_cast<const T*>(a.q) + u.row * a.q_sr + (h * a.group + u.g) * a.q_sh,
                u.lo, u.hi, tiles, slot_of, sm, o))
          continue;
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
        const QueryRow u = query_row(a, c, r0 + r);
        const bool sees = u.lo < u.hi;
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
                       static_cast<int32_t>(2 * blockIdx.x + 1), from, to};
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
// strips of 5 pieces x 256 columns, 63 MB: 15.5 us).
template <typename T, int DP, int W>
__global__ void __launch_bounds__(256) forward_join(AttnArgs a, ForwardPlan fp) {
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
    const size_t at = fp.decode ? (p == 0 ? hd.first : hd.first - 1 + 2 * static_cast<size_t>(p)) : hd.first + p;
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
    const bool sees = r >= hd.from && r < hd.to;
    T* to = reinterpret_cast<T*>(a.out) + row * a.o_sr + head * a.o_sh;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (lane * PER + i < a.d) to[lane * PER + i] = store_cvt<T>(sees ? o[i] / l : 0.f);
    if (a.lse && lane == 0) a.lse[row * a.hq + head] = sees ? (m2 + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
  }
}

}  // namespace

template <typename T, int DP>
hipError_t run_forward(const AttnArgs& a, const ForwardPlan& p, hipStream_t st) {
  constexpr Cap kPart = sizeof(T) == 2 ? Cap::part : Cap::tanh;
  const bool cap = a.cap2 != 0.f, part = a.cap2 <= static_cast<float>(kPartCap * kLog2e);
  auto* kernel = p.decode ? !cap   ? forward_decode<T, DP, Cap::none>
                            : part ? forward_decode<T, DP, kPart>
                                   : forward_decode<T, DP, Cap::tanh>
                 : !cap   ? forward_chunk<T, DP, Cap::none>
                 : part   ? forward_chunk<T, DP, kPart>
                          : forward_chunk<T, DP, Cap::tanh>;
  const dim3 block(p.decode ? 64 * Decode<T, DP>::kWaves : 256);
  const hipError_t e = launch_on(kernel, dim3(p.grid), block, st, a, p);
  if (p.splits == 1) return e;
  if (e != hipSuccess) return e;
  return p.decode ? launch_on(forward_join<T, DP, 4>, dim3(p.grid, p.join_rows), dim3(256), st, a, p)
                  : launch_on(forward_join<T, DP, 1>, dim3(p.strips * a.hkv, p.join_rows / 4), dim3(256), st, a, p);
}

template hipError_t run_forward<float, KVX_ATTN_DP>(const AttnArgs&, const ForwardPlan&, hipStream_t);
template hipError_t run_forward<bf16_t, KVX_ATTN_DP>(const AttnArgs&, const ForwardPlan&, hipStream_t);

}  // namespace kvx
