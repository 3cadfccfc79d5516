// attn_evict.hip -- keep the cached tokens of the largest weight
// (kvx_attn_evict): a selection per (layer, context, KV head), then the rows.
#include <algorithm>

#include "attn.h"

namespace kvx {
namespace {

constexpr int kSelThreads = 1024;

// A weight as an unsigned number of the same order; -0 as +0, NaN as -inf.
__device__ __forceinline__ uint32_t order_key(float f) {
  if (f != f) f = -INFINITY;
  const uint32_t u = __float_as_uint(f + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Exclusive sum of x over the workgroup in thread order; `total` the whole.
// One use of `sh` ends with a barrier.
__device__ __forceinline__ int block_scan(int x, int* sh, int& total) {
  const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
  int s = x;
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) {
    const int y = __shfl_up(s, i);
    if (lane >= i) s += y;
  }
  if (lane == 63) sh[w] = s;
  __syncthreads();
  int base = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < kSelThreads / 64; ++i) {
    const int y = sh[i];
    if (i < w) base += y;
    total += y;
  }
  __syncthreads();
  return base + s - x;
}

constexpr int kBins = 2048;
constexpr int kHeld = 8;                           // weights of a thread in registers
constexpr int kChunk = kHeld * kSelThreads;        // slots of the workgroup's
constexpr int kWaves = kSelThreads / 64;

// Positions in slot order of the slots that are on, where slot u * 1024 + t of
// a chunk is thread t's bit u: counts of every wave and u, then their sums
// before it; only the first `rounds` u have any.  `count` is the caller's for
// this use alone.  Returns the number of slots on.
__device__ __forceinline__ int chunk_scan(uint32_t on, int rounds, int* count, int (&at)[kHeld]) {
  const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
  if (lane >= rounds && lane < kHeld) count[lane * kWaves + w] = 0;
#pragma unroll
  for (int u = 0; u < kHeld; ++u) {
    if (u >= rounds) continue;
    const uint64_t m = __ballot(on >> u & 1);
    at[u] = __popcll(m & ((1ull << lane) - 1));
    if (lane == 0) count[u * kWaves + w] = __popcll(m);
  }
  __syncthreads();
  static_assert(kHeld * kWaves == 128, "two counts a lane");
  const int c0 = count[2 * lane], c1 = count[2 * lane + 1];
  int s = c0 + c1;
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) {
    const int y = __shfl_up(s, i);
    if (lane >= i) s += y;
  }
  const int before = s - c0 - c1;
#pragma unroll
  for (int u = 0; u < kHeld; ++u) {
    if (u >= rounds) continue;
    const int i = u * kWaves + w;
    at[u] += __shfl(before, i / 2) + (i % 2 ? __shfl(c0, i / 2) : 0);
  }
  return __shfl(s, 63);
}

// One workgroup per (layer, context, KV head).  The key of the last kept slot
// is found by a radix search over the keys' bits, 11, 11 and 10 at a time from
// the top (counts of the keys that share the prefix found so far); slots above
// it are kept, of those equal to it the first ones, and a scan in slot order
// writes the kept slots in rising order.  11 bits: the first hold sign,
// exponent and two bits of the number, so that counts of like weights fall on
// more than a few counters.  Up to 8192 slots the weights are read once and
// stay in registers; longer contexts are read again for each of the steps.
// Bound by latency: three rounds of LDS counters, their scan and the search (the
// last decides nothing where no two weights share the first 22 bits).
// Measured: 56 selections of 1024 of 2047 slots 11.8 us, 416 of 2048 of up to 8192
// 24 us.
__global__ void __launch_bounds__(kSelThreads, 8) evict_select(EvictArgs a) {
  __shared__ int count[kBins];
  __shared__ int counts[2][128];
  __shared__ int scan[kWaves];
  __shared__ int found[3];  // digit, rank left within it, its count
  const int set = a.set0 + blockIdx.x, tid = threadIdx.x;
  const int b = set / a.heads % a.batch;
  const int n = min(max(a.tokens[b], 0), a.src.capacity), weighed = min(n, a.mass_capacity);
  const int keep = min(n, a.keep);
  if (a.tokens_out && tid == 0 && set < a.heads * a.batch && set % a.heads == 0)
    a.tokens_out[b] = keep;
  const float* w = a.mass + static_cast<int64_t>(set) * a.mass_capacity;
  float* wo = a.mass_out ? a.mass_out + static_cast<int64_t>(set) * a.mass_capacity : nullptr;
  int32_t* kept = a.kept + static_cast<int64_t>(set) * a.keep;
  const int first = min(a.sink, n), last = max(first, n - a.recent);
  const int middle = keep - first - (n - last);  // slots to pick from [first, last)
  const bool all = keep == n, search = !all && middle > 0;
  const int chunks = (n + kChunk - 1) / kChunk;
  const int rounds = min(kHeld, (n + kSelThreads - 1) / kSelThreads);  // of a chunk
  float x[kHeld];
  auto load = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
      const int j = c * kChunk + u * kSelThreads + tid;
      x[u] = j < weighed ? w[j] : 0.f;
    }
  };
  if (chunks == 1) load(0);
  uint32_t key = 0;
  int equal = 0;      // of the keys equal to `key`, how many are kept
  bool some = false;  // and whether not all are
  if (search) {
    uint32_t mask = 0;
    int rank = middle;  // looking for the rank-th largest
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int bits = pass < 2 ? 11 : 10, shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      for (int i = tid; i < kBins; i += kSelThreads) count[i] = 0;
      __syncthreads();
      for (int c = 0; c < chunks; ++c) {
        if (chunks > 1) load(c);
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
          if (u >= rounds) continue;
          const int j = c * kChunk + u * kSelThreads + tid;
          const uint32_t k = order_key(x[u]);
          if (j >= first && j < last && (k & mask) == key)
            atomicAdd(&count[k >> shift & ((1u << bits) - 1)], 1);
        }
      }
      __syncthreads();
      // thread t: two counters from the top
      const int d = kBins - 2 - 2 * tid;
      const int hi = count[d + 1], lo = count[d];
      int total;
      const int above = block_scan(hi + lo, scan, total);
      if (above < rank && rank <= above + hi + lo) {
        const bool upper = rank <= above + hi;
        found[0] = upper ? d + 1 : d;
        found[1] = rank - above - (upper ? 0 : hi);
        found[2] = upper ? hi : lo;
      }
      __syncthreads();
      key |= static_cast<uint32_t>(found[0]) << shift;
      rank = found[1];
      some = rank < found[2];
      mask |= ((1u << bits) - 1) << shift;
    }
    equal = rank;
  }
  int done = 0, ties = 0;
  for (int c = 0; c < chunks; ++c) {
    if (chunks > 1) load(c);
    uint32_t on = 0, tie = 0;
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
      if (u >= rounds) continue;
      const int j = c * kChunk + u * kSelThreads + tid;
      const uint32_t k = order_key(x[u]);
      const bool picked = j >= first && j < last && !all;
      const bool same = k == key;
      if (picked ? search && (k > key || (same && !some)) : j < n) on |= 1u << u;
      if (picked && some && same) tie |= 1u << u;
    }
    int at[kHeld];
    if (some) {
      const int total = chunk_scan(tie, rounds, counts[0], at);
#pragma unroll
      for (int u = 0; u < kHeld; ++u)
        if ((tie >> u & 1) && ties + at[u] < equal) on |= 1u << u;
      ties += total;
    }
    const int total = chunk_scan(on, rounds, counts[1], at);
    // in place: this chunk's weights have all been read, a barrier ago
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
      if (on >> u & 1) {
        kept[done + at[u]] = c * kChunk + u * kSelThreads + tid;
        if (wo && done + at[u] < a.mass_capacity) wo[done + at[u]] = x[u];
      }
    done += total;
    __syncthreads();  // the counts' next use
  }
  for (int64_t i = keep + tid; i < a.keep; i += kSelThreads) kept[i] = -1;
  if (wo)
    for (int i = keep + tid; i < min(a.mass_capacity, max(a.keep, n)); i += kSelThreads) wo[i] = 0.f;
}

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;

constexpr int kMoveThreads = 256;
constexpr int kMoveUnroll = 8;  // 16-byte pieces of a thread in flight

// A workgroup per (layer, context, KV head), K|V and part of the rows' pieces
// (in place) or of the rows (elsewhere).  Steps of 256 x 8 pieces, all read
// before any is written.  In place that is safe for every later step too: kept
// slots rise, so row i comes from slot >= i.
// Bound by memory.  Measured: 26 layers, 4 contexts of up to 8192 slots to 2048,
// 4 heads x 256, pages of 32: 1761 MB in 370 to 410 us, 4.3 to 4.8 TB/s; 28 layers of
// 2047 to 1024, 2 heads x 128: 60 MB in 12 us.
__global__ void __launch_bounds__(kMoveThreads) evict_move(EvictArgs a, int log_pieces, int rows) {
  const int set = a.set0 + blockIdx.x, v = blockIdx.y, tid = threadIdx.x;
  const int h = set % a.heads, b = set / a.heads % a.batch, l = set / a.heads / a.batch;
  const int n = min(max(a.tokens[b], 0), a.src.capacity);
  const int keep = min(min(n, a.keep), a.dst.capacity);
  const int32_t* kept = a.kept + static_cast<int64_t>(set) * a.keep;
  const int pieces = 1 << log_pieces;
  const int per = a.row_bytes / 16 >> log_pieces;  // parts that a row is in
  const int p0 = blockIdx.z % per * pieces;
  const int r_first = blockIdx.z / per * rows;
  const int r_end = min(keep, a.in_place ? keep : r_first + rows);
  // the pointers by value: chosen by address they would be kept in memory
  const char *sk = a.src.k, *sv = a.src.v;
  char *dk = a.dst.k, *dv = a.dst.v;
  const char* src = (v ? sv : sk) + l * a.src.sl + h * a.src.sh;
  char* dst = (v ? dv : dk) + l * a.dst.sl + h * a.dst.sh;
  const int step = kMoveThreads * kMoveUnroll >> log_pieces;  // rows
  for (int r0 = r_first; r0 < r_end; r0 += step) {
    u32x4 x[kMoveUnroll];
    int64_t to[kMoveUnroll];
    bool on[kMoveUnroll];
#pragma unroll
    for (int u = 0; u < kMoveUnroll; ++u) {
      // past the end: the last row again, not stored
      const int i = u * kMoveThreads + tid, p = (p0 + (i & (pieces - 1))) * 16;
      const int r = min(r0 + (i >> log_pieces), r_end - 1), j = kept[r];
      on[u] = r0 + (i >> log_pieces) < r_end && !(a.in_place && j == r);
      to[u] = cache_offset(a.dst, cache_block(a.dst, b, r), r) + p;
      x[u] = *reinterpret_cast<const u32x4*>(src + cache_offset(a.src, cache_block(a.src, b, j), j) + p);
    }
    if (a.in_place) __syncthreads();
#pragma unroll
    for (int u = 0; u < kMoveUnroll; ++u)
      if (on[u]) *reinterpret_cast<u32x4*>(dst + to[u]) = x[u];
  }
}

// Strides in bytes.
CacheArgs in_bytes(CacheArgs c, int es) {
  c.sl *= es;
  c.sb *= es;
  c.sh *= es;
  c.st *= es;
  return c;
}

}  // namespace

hipError_t launch_evict(const kvx_attn* at, const EvictArgs& args, hipStream_t st) {
  EvictArgs a = args;
  const int es = at->dtype == KVX_F32 ? 4 : 2;
  a.src = in_bytes(a.src, es);
  a.dst = in_bytes(a.dst, es);
  const int sets = a.layers * a.batch * a.heads;
  // pieces of a workgroup: a power of two that divides a row's, of at least 128
  // bytes (a memory line).  Elsewhere a step of rows a workgroup, more where a
  // launch would have too many; rows past the cache's slots are never kept
  const int whole = a.row_bytes / 16;
  int pieces = whole & -whole, rows = std::min(a.keep, a.src.capacity), parts;
  if (a.in_place) {
    pieces = std::min(pieces, 8);
    parts = whole / pieces;
  } else {
    pieces = std::min(pieces, 64);
    const int most = rows, per = whole / pieces;
    rows = kMoveThreads * kMoveUnroll / pieces;
    while (per * ((int64_t(most) + rows - 1) / rows) > 65535) rows *= 2;
    parts = static_cast<int>(per * ((int64_t(most) + rows - 1) / rows));
  }
  // a launch has less than 2^32 threads along x
  constexpr int kMost = 1 << 21;
  for (a.set0 = 0; a.set0 < sets; a.set0 += kMost) {
    const int some = std::min(sets - a.set0, kMost);
    hipError_t e = launch_on(evict_select, dim3(some), dim3(kSelThreads), st, a);
    if (e == hipSuccess)
      e = launch_on(evict_move, dim3(some, 2, parts), dim3(kMoveThreads), st, a, __builtin_ctz(pieces), rows);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace kvx
