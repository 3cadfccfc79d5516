// attn_evict.hip -- keep the cached tokens of the largest weight
// (kvx_attn_evict): a selection per (layer, context, KV head), then the rows.
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

// One workgroup per (layer, context, KV head).  The key of the last kept slot
// is found by a radix search over the keys' bits, 8 at a time from the top
// (counts of the keys that share the prefix found so far); slots above it are
// kept, of those equal to it the first ones, and a scan in slot order writes
// the kept slots in rising order.
__global__ void __launch_bounds__(kSelThreads) evict_select(EvictArgs a) {
  __shared__ int count[256];
  __shared__ int scan[kSelThreads / 64];
  __shared__ uint32_t found[2];  // prefix, rank left within it
  const int set = blockIdx.x, tid = threadIdx.x;
  const int b = set / a.heads % a.batch;
  const int n = min(min(max(a.tokens[b], 0), a.src.capacity), a.mass_capacity);
  const int keep = min(n, a.keep);
  if (a.tokens_out && tid == 0 && set < a.heads * a.batch && set % a.heads == 0)
    a.tokens_out[b] = keep;
  const float* w = a.mass + static_cast<int64_t>(set) * a.mass_capacity;
  float* wo = a.mass_out ? a.mass_out + static_cast<int64_t>(set) * a.mass_capacity : nullptr;
  int32_t* kept = a.kept + static_cast<int64_t>(set) * a.keep;
  const int first = min(a.sink, n), last = max(first, n - a.recent);
  int middle = keep - first - (n - last);  // slots to pick from [first, last)
  const bool all = keep == n;
  uint32_t key = 0;
  int equal = 0;  // of the keys equal to `key`, how many are kept
  if (!all && middle > 0) {
    uint32_t prefix = 0, mask = 0;
    int rank = middle;  // looking for the rank-th largest
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kSelThreads) count[i] = 0;
      __syncthreads();
      for (int j = first + tid; j < last; j += kSelThreads) {
        const uint32_t k = order_key(w[j]);
        if ((k & mask) == prefix) atomicAdd(&count[k >> shift & 255], 1);
      }
      __syncthreads();
      if (tid == 0) {
        int d = 255, r = rank;
        while (d > 0 && count[d] < r) r -= count[d--];
        found[0] = prefix | static_cast<uint32_t>(d) << shift;
        found[1] = r;
      }
      __syncthreads();
      prefix = found[0];
      rank = found[1];
      mask |= 255u << shift;
    }
    key = prefix;
    equal = rank;
  }
  int done = 0, ties = 0;
  for (int j0 = 0; j0 < n; j0 += kSelThreads) {
    const int j = j0 + tid;
    const float x = j < n ? w[j] : 0.f;
    int total, tie = 0;
    bool keep_j = j < n;
    if (!all && j >= first && j < last) {
      const uint32_t k = order_key(x);
      tie = middle > 0 && k == key;
      keep_j = middle > 0 && k > key;
    }
    const int before = block_scan(tie, scan, total);
    if (tie) keep_j = ties + before < equal;
    ties += total;
    const int at = done + block_scan(keep_j, scan, total);
    if (keep_j) {
      kept[at] = j;
      // in place: slots up to j have all been read, a barrier ago
      if (wo) wo[at] = x;
    }
    done += total;
  }
  for (int i = keep + tid; i < a.keep; i += kSelThreads) kept[i] = -1;
  if (wo) {
    __syncthreads();
    for (int i = keep + tid; i < min(a.mass_capacity, max(a.keep, n)); i += kSelThreads) wo[i] = 0.f;
  }
}

constexpr int kMoveThreads = 256;

// One workgroup per (layer, context, KV head, K|V): kept rows in steps, each
// step's rows all read before any is written.  In place that is safe for every
// later step too: kept slots rise, so row i comes from slot >= i.
__global__ void __launch_bounds__(kMoveThreads) evict_move(EvictArgs a) {
  const int set = blockIdx.x, v = blockIdx.y, tid = threadIdx.x;
  const int h = set % a.heads, b = set / a.heads % a.batch, l = set / a.heads / a.batch;
  const int n = min(min(max(a.tokens[b], 0), a.src.capacity), a.mass_capacity);
  const int keep = min(min(n, a.keep), a.dst.capacity);
  const int32_t* kept = a.kept + static_cast<int64_t>(set) * a.keep;
  const int pieces = a.row_bytes / 16;
  const char* src = v ? a.src.v : a.src.k;
  char* dst = v ? a.dst.v : a.dst.k;
  const int64_t total = static_cast<int64_t>(keep) * pieces;
  for (int64_t i0 = 0; i0 < total; i0 += kMoveThreads) {
    const int64_t i = i0 + tid;
    const bool on = i < total;
    uint4 x{};
    const int r = static_cast<int>(i / pieces), p = static_cast<int>(i % pieces);
    if (on) {
      const int j = kept[r];
      const int64_t o = l * a.src.sl + h * a.src.sh + cache_offset(a.src, cache_block(a.src, b, j), j);
      x = *reinterpret_cast<const uint4*>(src + o + p * 16);
    }
    __syncthreads();
    if (on) {
      const int64_t o = l * a.dst.sl + h * a.dst.sh + cache_offset(a.dst, cache_block(a.dst, b, r), r);
      *reinterpret_cast<uint4*>(dst + o + p * 16) = x;
    }
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
  const hipError_t e = launch_on(evict_select, dim3(sets), dim3(kSelThreads), st, a);
  if (e != hipSuccess) return e;
  return launch_on(evict_move, dim3(sets, 2), dim3(kMoveThreads), st, a);
}

}  // namespace kvx
