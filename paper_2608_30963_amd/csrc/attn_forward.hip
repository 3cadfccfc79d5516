// attn_forward.hip -- attention of new tokens over the cache
// (kvx_attn_forward): which kernel a call runs, and its workspace.
#include "attn_forward.h"

#include <algorithm>

namespace kvx {
namespace {

int padded_dim(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

// Pieces that the units of the chunk kernel are split into, at most: with fewer
// workgroups than the compute units take some of those would idle.
int64_t most_pieces(const kvx_attn* at) { return 2 * int64_t(at->n_cu); }

// Workgroups of the chunk kernel that a compute unit takes at once.
int resident(const kvx_attn* at) {
  return padded_dim(at->model.head_dim) * (at->dtype == KVX_F32 ? 4 : 2) <= 256 ? 2 : 1;
}

// Pieces of a unit: each costs a share of the unit and some 3% of it to start
// and to join, and the card takes so many workgroups at a time.  Measured (us)
// unsplit, in 2, 4 and 5 pieces: 1531 tokens in 5627 slots, heads 8 / 4 x 256,
// capped, 100 units: 191, 116, 128, 120 (takes 5); fp32, 3 contexts of up to 257 in
// 1024, heads 12 / 2 x 128, 58 units: 153, 88, 56, 71 (takes 4).
int splits_of(const kvx_attn* at, int64_t units) {
  const int64_t slots = int64_t(at->n_cu) * resident(at);
  int best = 1;
  double least = 1e30;
  for (int s = 1; s <= 16 && (s == 1 || units * s <= most_pieces(at)); ++s) {
    const double cost = double((units * s + slots - 1) / slots) * (1.0 / s + 0.03);
    if (cost < least) {
      least = cost;
      best = s;
    }
  }
  return best;
}

size_t head_bytes(const kvx_attn* at) { return (most_pieces(at) * sizeof(JoinHead) + 255) / 256 * 256; }

}  // namespace

size_t forward_workspace(const kvx_attn* at) {
  const int dp = padded_dim(at->model.head_dim);
  return head_bytes(at) + most_pieces(at) * piece_floats(kChunkRows, dp) * sizeof(float);
}

hipError_t launch_forward(const kvx_attn* at, const AttnArgs& a, int max_new, void* workspace,
                          hipStream_t st) {
  ForwardPlan p{};
  p.heads = static_cast<JoinHead*>(workspace);
  p.pieces = reinterpret_cast<float*>(static_cast<char*>(workspace) + head_bytes(at));
  // up to 32 query rows per context: the ring of single tokens, which splits the
  // cache evenly over the card; more: the chunk kernel.  Measured (us; ring,
  // chunk), heads 28 / 4 x 128, 16 contexts of 4096 slots: 28 rows 36.6, 36.1; 56
  // rows 54.4, 44.0; 112 rows 83.0, 56.6; one of 128k: 7 rows 53, 239; 28 rows 62,
  // 241.  A few contexts of 1024 slots lose by it: 28 rows 18.7, 15.0.
  const int64_t strips = (int64_t(a.rows) * at->group + kChunkRows - 1) / kChunkRows +
                         std::min(a.batch, a.rows);
  const int64_t units = strips * a.hkv;
  p.decode = int64_t(max_new) * at->group <= kDecodeRows || !launchable(units, 256);
  if (p.decode) {
    p.grid = at->n_cu;
    p.splits = 0;  // as many as the lengths give
    // caches of few slots (the host knows no lengths): a workgroup a unit, no
    // join.  Measured (us, captured;
    // split, whole), heads 12 / 2: 128 slots 10.5, 7.5; 512 10.9, 11.4; 1024 11.5,
    // 16.8; 64 contexts of 300 slots, heads 64 / 8: 29.0, 25.8; 32 of 1024, heads
    // 28 / 4: 21.2, 21.6
    if (a.c.capacity <= 512) p.splits = 1;
    p.join_rows = static_cast<int>(std::min(int64_t(max_new) * at->group, int64_t(kDecodeRows)));
  } else {
    p.join_rows = kChunkRows;
    p.splits = splits_of(at, units);
    p.strips = static_cast<int>(strips);
    p.grid = static_cast<int>(units * p.splits);
  }
  const bool f32 = at->dtype == KVX_F32;
  switch (padded_dim(at->model.head_dim)) {
    case 64: return f32 ? run_forward<float, 64>(a, p, st) : run_forward<bf16_t, 64>(a, p, st);
    case 128: return f32 ? run_forward<float, 128>(a, p, st) : run_forward<bf16_t, 128>(a, p, st);
    default: return f32 ? run_forward<float, 256>(a, p, st) : run_forward<bf16_t, 256>(a, p, st);
  }
}

}  // namespace kvx
