// attn_mass_d.hip -- the attention-weight kernels of one padded head_dim
// (KVX_ATTN_DP = 64, 128 or 256), both dtypes.
//
// A lane holds one slot's scores with 16 query rows, so a slot's weight is a
// sum over its registers and the other half's; no two workgroups add to one
// slot, and the order of the sum is fixed.  The weight of a score is
// exp2(score - lse), with the caller's log-sum-exp.
#include "attn_mass.h"
#include "attn_tile.h"

namespace kvx {
namespace {

// Slots past the cached tokens: mass_in's values, or zeros.
__device__ __forceinline__ void copy_rest(const AttnArgs& a) {
  if (a.mass_in == a.mass) return;
  for (int i = blockIdx.x; i < a.batch * a.hkv; i += gridDim.x) {
    const int n = min(max(a.tokens[i / a.hkv], 0), a.c.capacity);
    const int64_t at = static_cast<int64_t>(i) * a.mass_capacity;
    // eight values a thread at a time, for the latency of reading them
    for (int j0 = n + threadIdx.x; j0 < a.mass_capacity; j0 += 8 * blockDim.x) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int j = j0 + u * blockDim.x;
        x[u] = a.mass_in && j < a.mass_capacity ? a.mass_in[at + j] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int j = j0 + u * blockDim.x;
        if (j < a.mass_capacity) a.mass[at + j] = x[u];
      }
    }
  }
}

// exp2(score - lse) of one score: `less` is -lse in log2 units, -inf for rows
// that are not there.  Weights are fp32 whatever the keys are, so capped scores
// are formed by the tanh of relative precision.
template <bool CAP>
__device__ __forceinline__ float weight_of(const AttnArgs& a, float x, float less) {
  return __builtin_amdgcn_exp2f(CAP ? __builtin_fmaf(a.cap2, cap_tanh(a, x), less)
                                    : __builtin_fmaf(x, a.scale2, less));
}

// Sum of the weights of the lane's slot over its 16 rows.  Where every score of the
// wave is less than half its cap, which is the rule, a polynomial alone serves.
// Measured (us, a few calls in a row; with it, without it, and by 1 - 2 / (1 + exp
// 2y), whose error in a weight was ten times as large), cap 50: 1021 tokens over 8k
// slots, heads 8 / 4 x 256: 68, 80, 66; 1024 over 8k, heads 28 / 4 x 128: 169, 203,
// 155; 64 contexts of single tokens over up to 4k slots, heads 8 / 4 x 256: 69, 74, -.
template <bool CAP>
__device__ __forceinline__ float weigh(const AttnArgs& a, const f32x16& s, const float (&less)[16]) {
  float sum[2] = {0.f, 0.f};
  if constexpr (CAP) {
    float top = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) top = fmaxf(top, fabsf(s[v]));
    if (!__any(!(top < a.near))) {
#pragma unroll
      for (int v = 0; v < 16; ++v) sum[v % 2] += __builtin_amdgcn_exp2f(cap_near(a, s[v], less[v]));
      return sum[0] + sum[1];
    }
  }
#pragma unroll
  for (int v = 0; v < 16; ++v) sum[v % 2] += weight_of<CAP>(a, s[v], less[v]);
  return sum[0] + sum[1];
}

// The same where rows may not see the lane's slot j; r0 is the first row.
template <bool CAP>
__device__ __forceinline__ float weigh_seen(const AttnArgs& a, const Context& c, const f32x16& s,
                                            const float (&less)[16], int r0, int j) {
  const int h = threadIdx.x % 64 / 32;
  float sum = 0.f;
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const QueryRow q = query_row(a, c, r0 + 8 * (v / 4) + 4 * h + v % 4);
    const float p = weight_of<CAP>(a, s[v], less[v]);
    if (j >= q.lo && j < q.hi) sum += p;
  }
  return sum;
}

// ---------------------------------------------------------------------------
// Single tokens (and few): the query rows in registers, the slots streamed
// through the waves' own rings.  Bound by memory: keys are read once, the line
// of all work is cut into equal ranges as in forward's single tokens.  Measured:
// 64 contexts of up to 4k slots, heads 28 / 4 x 128, 156 MB in 52 us, the kernel
// 42 us (3.7 TB/s), of which about 10 pass before the first keys arrive: mass_in
// past the tokens, which the keys could be asked for ahead of, lengths of 64
// contexts, block numbers.
// ---------------------------------------------------------------------------

template <typename T, int DP, bool CAP>
__global__ void __launch_bounds__((64 * ring_waves(32 * DP * sizeof(T))), 1) mass_decode(AttnArgs a) {
  using L = Tile<T, DP>;
  constexpr int kStage = 32 * L::kRowBytes;
  constexpr int NW = ring_waves(kStage), NST = ring_stages(kStage);
  constexpr int kCopies = kStage / 1024, kStep = NW * 32;
  __shared__ __attribute__((aligned(16))) char lds[NW * NST * kStage];
  __shared__ float earlier[NW][NST][32];  // mass_in of the rings' tiles
  const int lane = threadIdx.x % 64, n = lane % 32, half = lane / 32;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  copy_rest(a);
  const Share share = line_share(a, [&](int b) {
    const int n = min(max(a.tokens[b], 0), min(a.c.capacity, a.mass_capacity));
    return static_cast<int64_t>((n + kStep - 1) / kStep);
  });
  if (share.s0 >= share.s1) return;
  int h = share.h, b = share.b, step = share.step;
  char* const ring = lds + w * NST * kStage;
  const uint32_t ring3 = lds_address(lds) + w * NST * kStage;
  const typename L::LaneAt at = L::lane_at();
  if (a.d < DP) {
    for (int i = lane; i < NST * kStage / 16; i += 64)
      reinterpret_cast<uint4*>(ring)[i] = uint4{0, 0, 0, 0};
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
  for (int64_t s = share.s0; s < share.s1;) {
    const Context c = context(a, b);
    const int end = min(c.n, a.mass_capacity);  // slots that are written
    const int all = (end + kStep - 1) / kStep;
    const int cnt = static_cast<int>(min<int64_t>(all - step, share.s1 - s));
    const char* kb = a.c.k + h * a.c.sh * static_cast<int64_t>(sizeof(T));
    const int j_first = (step * NW + w) * 32;
    const int64_t mrow = (static_cast<int64_t>(b) * a.hkv + h) * a.mass_capacity;
    const int tiles = min(cnt, end > j_first ? (end - j_first + kStep - 1) / kStep : 0);
    auto slot_of = [&](int t) __attribute__((always_inline)) { return j_first + t * kStep; };
    for (int r0 = 0; r0 == 0 || r0 < c.m * a.group; r0 += 32) {
      // rows of this pass (one, if the caller's bound on new tokens holds):
      // what they see together, and all of them
      const int valid = min(32, c.m * a.group - r0);
      int lo = 0, hi = 0, alo = 0, ahi = 0, x;
      if (valid > 0) {
        seen_by(a, c, r0, r0 + valid - 1, lo, hi);
        seen_by(a, c, r0, r0, x, ahi);
        seen_by(a, c, r0 + valid - 1, r0 + valid - 1, alo, x);
      }
      const QueryRow qr = query_row(a, c, r0 + n);
      uint4 q[L::kQ];
      const T* qp = reinterpret_cast<const T*>(a.q) + qr.row * a.q_sr + (h * a.group + qr.g) * a.q_sh;
      L::load_q(q, n < valid ? qp : nullptr, a.d);
      float less[16];
      int first, last;
      seeing(a, c, r0, first, last);
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int r = 8 * (v / 4) + 4 * half + v % 4, i = fdiv(a.by_group, r0 + r);
        less[v] = r >= first && r < last
                      ? -kLog2e * a.lse[static_cast<int64_t>(c.q0 + i) * a.hq + h * a.group +
                                        (r0 + r - i * a.group)]
                      : -INFINITY;
      }
      // tiles that the rows see: from t0 to t1; the others keep their sums
      const int t0 = hi > lo && lo > j_first + 31 ? (lo - j_first - 32) / kStep + 1 : 0;
      const int t1 = hi > lo ? min(tiles, hi > j_first ? (hi - j_first + kStep - 1) / kStep : 0) : 0;
      Blocks<32> blocks;
      const float* from = r0 > 0 ? a.mass : a.mass_in;
      const uint32_t earlier3 = lds_address(reinterpret_cast<const char*>(earlier[w]));
      auto copy = [&](int t) __attribute__((always_inline)) {
        if (from && lane < 32)
          copy4(reinterpret_cast<const char*>(from + mrow + min(slot_of(t) + n, end - 1)),
                earlier3 + t % NST * 128);
        copy_tile<T, DP, 32, 1, true, false>(a.c, kb, nullptr, b, slot_of(t), lo, hi, blocks, a.d, 0,
                                             ring3 + t % NST * kStage, 0);
      };
      auto put = [&](int t, float sum) __attribute__((always_inline)) {
        const int j = slot_of(t) + n;
        if (lane < 32 && j < end) a.mass[mrow + j] = sum;
      };
      if (r0 == 0 && a.mass_in != a.mass)
        for (int t = 0; t < tiles; ++t)
          if (t < t0 || t >= t1)
            put(t, a.mass_in ? a.mass_in[mrow + min(slot_of(t) + n, end - 1)] : 0.f);
      if (t0 < t1) fetch_blocks(a.c, b, slot_of(t0), hi, blocks);
      for (int t = t0; t < t0 + NST - 1 && t < t1; ++t) {
        copy(t);
        fetch_blocks(a.c, b, slot_of(t + 1), hi, blocks);
      }
      // the queries are here: the compiler must not wait for them in the loop
      __builtin_amdgcn_s_waitcnt(0);
      for (int t = t0; t < t1; ++t) {
        // the stage that tile t + NST - 1 takes was read a tile ago, its values
        // used before this line
        __builtin_amdgcn_sched_barrier(0);
        if (t + NST - 1 < t1) {
          copy(t + NST - 1);
          vm_wait<(NST - 1) * kCopies>();
        } else {
          vm_wait<0>();
        }
        const int j0 = slot_of(t);
        const f32x16 sc = L::template scores<true>(ring + t % NST * kStage, at, q);
        const float sum = half_sum(j0 >= alo && j0 + 32 <= ahi
                                       ? weigh<CAP>(a, sc, less)
                                       : weigh_seen<CAP>(a, c, sc, less, r0, j0 + n));
        put(t, (from ? earlier[w][t % NST][n] : 0.f) + sum);
        __builtin_amdgcn_sched_barrier(0);
        fetch_blocks(a.c, b, slot_of(t + NST), hi, blocks);
      }
      vm_wait<0>();  // the next pass reads these sums
    }
    s += cnt;
    step = 0;
    if (s < share.s1) {
      do {
        if (++b == a.batch) {
          b = 0;
          ++h;
        }
      } while (a.tokens[b] <= 0);
      b = __builtin_amdgcn_readfirstlane(b);
      h = __builtin_amdgcn_readfirstlane(h);
    }
  }
}

// ---------------------------------------------------------------------------
// Chunks: 8 waves, QW of them over the query rows and 8 / QW over the slots,
// 32 each.  The slots' keys stay in registers; stages of 32 QW query rows and
// their log-sum-exps are copied into LDS as many stages ahead of their use as
// 128 KB hold: a stage is less work than a copy's latency.  No slot is
// split over workgroups, so sums need no atomics and no second launch.  Bound by
// the matrix units and the weights' arithmetic in turn, which a barrier a stage
// keeps in step.  Measured: 1021 tokens in 8192 slots, heads 8 / 4 x 256,
// capped: 59 us, 545 TFLOP/s.
// ---------------------------------------------------------------------------

template <typename T, int DP, bool CAP, int QW>
__global__ void __launch_bounds__(512, DP * sizeof(T) <= 256 ? 2 : 1) mass_chunk(AttnArgs a, int blocks_per) {
  using L = Tile<T, DP>;
  constexpr int KW = 8 / QW, kRows = 32 * QW, kBytes = kRows * L::kRowBytes;
  constexpr int kCopies = kBytes / 1024 / 8;  // of a wave
  constexpr int kBuffers = 131072 / kBytes < 4 ? 131072 / kBytes : 4;
  constexpr int R = L::kRowsPerCopy;
  __shared__ __attribute__((aligned(16))) char lds[kBuffers * kBytes];
  __shared__ __attribute__((aligned(16))) float lse[kBuffers][kRows];
  const int lane = threadIdx.x % 64, n = lane % 32, half = lane / 32;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int qw = w % QW, kw = w / QW;
  copy_rest(a);
  // (context, head, slots): later slots are seen by fewer rows
  const int id = xcd_remap(blockIdx.x, gridDim.x);
  const int b = id / (a.hkv * blocks_per), h = id / blocks_per % a.hkv;
  const int j_first = id % blocks_per * (KW * 32);
  const Context c = context(a, b);
  const int end = min(c.n, a.mass_capacity);  // slots that are written
  if (j_first >= end) return;
  const int j_last = min(end, j_first + KW * 32) - 1;
  // rows of the tokens that see any of the workgroup's slots
  const int p0 = c.p0;
  const int i0 = max(max(0, -p0), j_first < c.prefix ? 0 : j_first - p0);
  // (not below 0: a negative count times the heads may pass 32 bits)
  const int i1 =
      a.window ? static_cast<int>(max<int64_t>(0, min<int64_t>(c.m, int64_t(j_last) + a.window - p0))) : c.m;
  const int r_first = i0 * a.group, r_end = i1 * a.group;
  const int stages = r_end > r_first ? (r_end - r_first + kRows - 1) / kRows : 0;

  const int j = j_first + kw * 32 + n;
  uint4 key[L::kQ];
  {
    const int jc = min(j, c.n - 1);
    // slots that no row sees may lie in blocks that are gone
    const bool seen = stages > 0 && j < c.n && (!a.window || j > p0 + i0 - a.window);
    const T* kp = reinterpret_cast<const T*>(a.c.k) + h * a.c.sh;
    if (seen) kp += cache_offset(a.c, cache_block(a.c, b, jc), jc);
    L::load_q(key, seen ? kp : nullptr, a.d);
  }
  const typename L::LaneAt at = L::lane_at();
  if (a.d < DP) {
    for (int i = threadIdx.x; i < kBuffers * kBytes / 16; i += 512)
      reinterpret_cast<uint4*>(lds)[i] = uint4{0, 0, 0, 0};
  }
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  const uint32_t l3 = lds_address(lds), lse3 = lds_address(reinterpret_cast<const char*>(lse));
  auto copy_stage = [&](int s, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int row = (i * 8 + w) * R + lane / L::kChunks;
      const int r = min(r_first + s * kRows + row, c.m * a.group - 1);
      const int chunk = (lane % L::kChunks) ^ L::key_swz(row);
      const int tok = fdiv(a.by_group, r), g = r - tok * a.group;
      const char* from = a.q + ((c.q0 + tok) * a.q_sr + (h * a.group + g) * a.q_sh) * static_cast<int64_t>(sizeof(T)) + chunk * 16;
      if (chunk * 16 < a.d * static_cast<int>(sizeof(T)))
        copy16(from, l3 + buf * kBytes + (i * 8 + w) * 1024);
    }
    if (w * 64 < kRows) {
      const int row = w * 64 + lane;
      const int r = min(r_first + s * kRows + row, c.m * a.group - 1);
      const int tok = fdiv(a.by_group, r), g = r - tok * a.group;
      copy4(reinterpret_cast<const char*>(a.lse + static_cast<int64_t>(c.q0 + tok) * a.hq + h * a.group + g),
            lse3 + (buf * kRows + w * 64) * 4);
    }
  };
  float sum = 0.f;
  for (int s = 0; s < kBuffers - 1 && s < stages; ++s) copy_stage(s, s);
  for (int s = 0; s < stages; ++s) {
    const int buf = s % kBuffers;
    // this stage has landed, kBuffers - 2 more may be in flight, and every wave
    // is done with the one before
    if (s + kBuffers - 2 < stages)
      vm_wait<(kBuffers - 2) * kCopies>();
    else
      vm_wait<0>();
    tile_barrier();
    if (s + kBuffers - 1 < stages) copy_stage(s + kBuffers - 1, (s + kBuffers - 1) % kBuffers);
    const int r0 = r_first + s * kRows + qw * 32;
    if (r0 >= r_end) continue;
    float less[16];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const f32x4 y = *reinterpret_cast<const f32x4*>(&lse[buf][qw * 32 + 8 * x + 4 * half]);
#pragma unroll
      for (int e = 0; e < 4; ++e) less[4 * x + e] = -kLog2e * y[e];
    }
    const f32x16 sc = L::template scores<false, 4>(lds + buf * kBytes + qw * 32 * L::kRowBytes, at, key);
    // whether all 32 rows see all of the wave's slots
    const int ja = j_first + kw * 32;
    int alo, ahi, x;
    seen_by(a, c, r0, r0, x, ahi);
    seen_by(a, c, min(r0 + 31, c.m * a.group - 1), min(r0 + 31, c.m * a.group - 1), alo, x);
    if (ja >= alo && ja + 32 <= ahi && r0 + 32 <= c.m * a.group)
      sum += weigh<CAP>(a, sc, less);
    else
      sum += weigh_seen<CAP>(a, c, sc, less, r0, j);
  }
  sum = half_sum(sum);
  // the row waves' sums, in their order
  float* red = reinterpret_cast<float*>(lds);
  tile_barrier();
  if (lane < 32) red[w * 32 + n] = sum;
  tile_barrier();
  if (qw == 0 && lane < 32 && j < end) {
    float all = 0.f;
#pragma unroll
    for (int i = 0; i < QW; ++i) all += red[(kw * QW + i) * 32 + n];
    const int64_t to = (static_cast<int64_t>(b) * a.hkv + h) * a.mass_capacity + j;
    a.mass[to] = (a.mass_in ? a.mass_in[to] : 0.f) + all;
  }
}

// Workgroups of a context and head.
template <int QW>
int chunk_groups(const AttnArgs& a) {
  constexpr int slots = 8 / QW * 32;
  return (std::min(a.mass_capacity, a.c.capacity) + slots - 1) / slots;
}

template <typename T, int DP, int QW>
hipError_t run_chunk(const AttnArgs& a, hipStream_t st) {
  const int per = chunk_groups<QW>(a);
  const int64_t grid = static_cast<int64_t>(per) * a.batch * a.hkv;
  return a.cap2 != 0.f
             ? launch_on(mass_chunk<T, DP, true, QW>, dim3(static_cast<unsigned>(grid)), dim3(512), st, a, per)
             : launch_on(mass_chunk<T, DP, false, QW>, dim3(static_cast<unsigned>(grid)), dim3(512), st, a, per);
}

}  // namespace

template <typename T, int DP>
hipError_t run_mass(const AttnArgs& a, bool decode, int n_cu, hipStream_t st) {
  // workgroups go by the capacity, which may be reserved far beyond the tokens: those
  // that no launch takes are left to the ring, which goes by the tokens
  if (decode || !launchable(static_cast<int64_t>(chunk_groups<2>(a)) * a.batch * a.hkv, 512)) {
    const dim3 block(64 * ring_waves(32 * DP * sizeof(T)));
    return a.cap2 != 0.f ? launch_on(mass_decode<T, DP, true>, dim3(n_cu), block, st, a)
                         : launch_on(mass_decode<T, DP, false>, dim3(n_cu), block, st, a);
  }
  // as many row waves as two buffers of their stages leave room for, where
  // workgroups of two row waves (128 slots) would leave compute units idle.
  // Measured (us; 2 row waves, most), by the number of such workgroups: 256
  // tokens in 1024 slots, heads 12 / 2 x 128, 18: 33, 15; 512 in 8192, 130: 53, 45;
  // heads 8 / 4 x 256, 512 in 4096, 132: 29, 21; 4 contexts of 512 in 8192, 1040:
  // 107, 154; heads 12 / 2 x 128, 520: 81, 175
  constexpr int most = DP * sizeof(T) <= 256 ? 8 : DP * sizeof(T) <= 512 ? 4 : 2;
  const int64_t wide = static_cast<int64_t>(a.c.capacity / 128 + 1) * a.batch * a.hkv;
  if (most > 2 && wide < n_cu) return run_chunk<T, DP, most>(a, st);
  return run_chunk<T, DP, 2>(a, st);
}

template hipError_t run_mass<float, KVX_ATTN_DP>(const AttnArgs&, bool, int, hipStream_t);
template hipError_t run_mass<bf16_t, KVX_ATTN_DP>(const AttnArgs&, bool, int, hipStream_t);

}  // namespace kvx
