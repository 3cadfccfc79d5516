// attn_forward.h -- the attention kernels' launchers, one translation unit per
// head_dim (attn_forward_d.hip, attn_view_d.hip), and the partial results that
// they share.
#pragma once

#include "attn_view.h"

namespace kvx {

// Partial results of a piece of a unit (32 or 128 query rows of a KV head):
// [rows] pairs (reference m2, sum l), then [rows][DP] sums, fp32.
__host__ __device__ inline size_t piece_floats(int rows, int dp) {
  return static_cast<size_t>(rows) * (dp + 2);
}

// A unit whose pieces have to be joined.
struct JoinHead {
  int32_t pieces;  // 0: nothing to join
  int32_t rows;    // valid query rows
  int32_t row0;    // row of the new tokens that query row 0 belongs to
  int32_t g0;      // its head within the group
  int32_t h;       // KV head
  int32_t first;   // index of the unit's first piece
  int32_t from, to;  // query rows that see anything
  int32_t b;         // context
  int32_t step;      // chunk: from one piece's index to the next one's
};

constexpr int kChunkRows = 128;  // query rows of a workgroup of the chunk kernel
constexpr int kDecodeRows = 32;
constexpr int kFewRows = 16;

// Workgroups of forward_few that a compute unit takes at once, by the padded
// head_dim and a number's bytes: two, so that one's start and joins pass beside
// the other's copies, where LDS has room for both.
constexpr int few_groups(int dp, int bytes) { return dp * bytes <= 256 ? 2 : 1; }

struct ForwardPlan {
  bool decode;
  bool few;       // decode, of up to kFewRows query rows: forward_few
  int grid;       // workgroups
  int splits;     // pieces of a unit; 1: none is split; decode: 0, as the work divides
  int strips;     // chunk: q tiles of all contexts, at most
  int join_rows;  // query rows that a unit has by the caller's bound
  JoinHead* heads;
  float* pieces;
};

template <typename T, int DP>
hipError_t run_forward(const AttnArgs& a, const ForwardPlan& p, hipStream_t st);
template <typename S, int DP>
hipError_t run_view(const AttnView& a, const ForwardPlan& p, hipStream_t st);

}  // namespace kvx
