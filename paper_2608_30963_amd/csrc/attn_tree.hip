// attn_tree.hip -- drafted trees: what each node sees (kvx_attn_tree), and the
// accepted path's move to the front (kvx_attn_accept).
#include <algorithm>

#include "attn_view.h"

namespace kvx {
namespace {

constexpr int kMostNodes = 64 * 32;  // of a context: kvx_tree_io.words is at most 64

// A workgroup a context.  A node's ancestors have falling indices, so one walk
// up its path fills its words from the last to the first.  Bound by the launch and
// the paths' length: 8 trees of 64 nodes 5 us, one of 16 2.4.
__global__ void __launch_bounds__(256) tree_kernel(TreeArgs a) {
  __shared__ int32_t up[kMostNodes];
  const int b = blockIdx.x;
  const int q0 = a.q_start ? min(max(a.q_start[b], 0), a.rows) : b;
  const int q1 = a.q_start ? min(max(a.q_start[b + 1], q0), a.rows) : b + 1;
  const int m = q1 - q0, nodes = min(m, a.words * 32);
  const int p0 = min(max(a.tokens[b], 0), INT32_MAX - 1024) - m;
  for (int i = threadIdx.x; i < nodes; i += 256) {
    const int p = a.parent[q0 + i];
    up[i] = p >= 0 && p < i ? p : -1;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < m; i += 256) {
    const int64_t row = static_cast<int64_t>(q0) + i;
    // how far the path leads is known before it is walked only for a window's sinks
    int depth = 0;
    if (a.window > 0 && i < nodes)
      for (int k = up[i]; k >= 0; k = up[k]) ++depth;
    uint32_t* mask = a.mask + row * a.words;
    int word = a.words - 1, before = 0;
    uint32_t bits = 0;
    for (int k = i < nodes ? i : -1; k >= 0; ++before, k = up[k]) {
      while (word > k >> 5) {
        mask[word--] = bits;
        bits = 0;
      }
      if (a.window == 0 || before < a.window || p0 + depth - before < a.sink) bits |= 1u << (k & 31);
    }
    for (; word >= 0; --word, bits = 0) mask[word] = bits;
    depth = max(before - 1, 0);
    if (a.depth) a.depth[row] = depth;
    if (a.pos) {
      const int pos = p0 + depth + (a.shift ? a.shift[b] : 0);
      for (int x = 0; x < a.axes; ++x) a.pos[static_cast<int64_t>(x) * a.rows + row] = pos;
    }
  }
}

// A workgroup a (layer, context, KV head).  As paths rise, a row moves to a slot
// that is not past its own, and not past any later row's: rows go in turns, each
// read by all of the workgroup before it is written.  Bound by latency, a chain of
// length, path, block and row a turn: 28 layers x 2 heads, one path 3.6 us; 26 layers x
// 32 contexts x 4 heads x 256 in e4m3 10.9.
__global__ void __launch_bounds__(256) accept_kernel(AcceptArgs a) {
  const int64_t sets = static_cast<int64_t>(a.layers) * a.batch * a.heads;
  const int pieces = a.row_bytes / 16, both = 2 * pieces;
  const int per = 256 / both;  // rows a turn, keys and values
  for (int64_t set = blockIdx.x; set < sets; set += gridDim.x) {
    const int h = static_cast<int>(set % a.heads);
    const int64_t lb = set / a.heads;
    const int b = static_cast<int>(lb % a.batch);
    const int64_t l = lb / a.batch;
    const int m = a.q_start ? max(a.q_start[b + 1] - a.q_start[b], 0) : 1;
    const int all = min(max(a.tokens[b], 0), INT32_MAX - 1024), p0 = all - m;
    const int count = min(min(max(a.count[b], 0), m), a.max_path);
    if (l == 0 && h == 0 && threadIdx.x == 0 && a.tokens_out) a.tokens_out[b] = p0 + count;
    const int sub = threadIdx.x / both, piece = threadIdx.x % both;
    char* base = (piece < pieces ? a.c.k : a.c.v) + (l * a.c.sl + h * a.c.sh) * a.es + piece % pieces * 16;
    for (int i0 = 0; i0 < count; i0 += per) {
      const int i = i0 + sub;
      bool moves = sub < per && i < count;
      int from = 0, to = 0;
      if (moves) {
        const int k = a.path[static_cast<int64_t>(b) * a.max_path + i];
        from = p0 + k;
        to = p0 + i;
        moves = k >= 0 && k < m && k != i && to >= 0 && from < a.c.capacity && from >= 0 && to < a.c.capacity;
      }
      uint4 x{};
      uint32_t pair = 0;
      int64_t pat = 0;
      char* dst = nullptr;
      if (moves) {
        const int32_t fb = cache_block(a.c, b, from), tb = cache_block(a.c, b, to);
        x = *reinterpret_cast<const uint4*>(base + cache_offset(a.c, fb, from) * a.es);
        dst = base + cache_offset(a.c, tb, to) * a.es;
        if (a.scale.p && piece == 0) {
          const auto slot = [&](int j) { return a.c.table ? j - fdiv(a.c.bs, j) * static_cast<int>(a.c.bs.d) : j; };
          const int64_t at = l * a.scale.sl + h * a.scale.sh;
          pair = a.scale.p[at + fb * a.scale.sb + slot(from) * a.scale.st];
          pat = at + tb * a.scale.sb + slot(to) * a.scale.st;
        }
      }
      __syncthreads();
      if (moves) {
        *reinterpret_cast<uint4*>(dst) = x;
        if (a.scale.p && piece == 0) a.scale.p[pat] = pair;
      }
      __syncthreads();
    }
  }
}

}  // namespace

hipError_t launch_tree(const TreeArgs& a, hipStream_t st) {
  return launch_on(tree_kernel, dim3(a.batch), dim3(256), st, a);
}

hipError_t launch_accept(const kvx_attn* at, const AcceptArgs& a, hipStream_t st) {
  const int64_t sets = static_cast<int64_t>(a.layers) * a.batch * a.heads;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(sets, 64 * int64_t(at->n_cu))));
  return launch_on(accept_kernel, grid, dim3(256), st, a);
}

}  // namespace kvx
