// Host rules of the head norm and of the gated delta rule: how work is cut, and what a workspace holds.
#pragma once
#include "tac_product_plan.h"

namespace tac {

// ---- head norm -----------------------------------------------------------------------------------

// Lanes that share a head.  Each holds up to four pairs of features: rotated ones from the first lane on and the others from a lane of their own on, so that a lane's first and its second
// features are neighbours each; only where that takes more than 64 lanes does a lane hold some of both.
struct HeadLanes {
  int lanes, apart;                  // apart: rotated pairs and others on lanes of their own
};
inline HeadLanes head_lanes(int D, int rotated) {
  const auto room = [](int n) { return n <= 8 ? 8 : n <= 16 ? 16 : n <= 32 ? 32 : 64; };
  const int apart = (rotated + 3) / 4 + (D / 2 - rotated + 3) / 4;
  return apart <= 64 ? HeadLanes{room(apart), 1} : HeadLanes{64, 0};
}

// Slices of a row's heads: the lanes of a slice take every `slices`-th head and turn them all by the angles that they have formed once.  As few slices as
// give every compute unit four workgroups of 256 lanes (16 rows of 24 heads of 128 bf16: 6.9 us, in one slice a row 15.0; 300 rows of 12: 6.9, 12.2).
inline int head_slices(int64_t rows, int heads, int lanes) {
  const int64_t wanted = (int64_t)kFittedUnits * 4 * (256 / lanes);
  const int64_t slices = (wanted + rows - 1) / rows;
  return (int)(slices < 1 ? 1 : slices > heads ? heads : slices);
}

// Workgroups of a launch; what they do not reach in one turn they take in further ones, whose loads are on their way while the heads before are worked on
// (65536 rows of 18 heads of 128 bf16: 141 us, a quarter of the workgroups 149, four times as many 142).
constexpr int64_t kHeadGroups = 16 * kFittedUnits;
inline int64_t head_groups(int64_t rows, int slices, int lanes, int64_t most) {
  const int64_t units = rows * slices, each = 256 / lanes;
  const int64_t groups = (units + each - 1) / each;
  return groups < most ? groups : most;
}
// the backward pass keeps the gains' gradients of a workgroup, 2 D numbers, in a row of the workspace
constexpr int64_t kHeadBackwardGroups = 3 * kFittedUnits;      // as many as are there at once (131 registers): 16384 x 24 x 128 bf16 122 -> 115 us

// ---- gated delta rule ------------------------------------------------------------------------------

inline int64_t delta_chunks(int64_t T) { return (T + TAC_DELTA_CHUNK - 1) / TAC_DELTA_CHUNK; }

// Columns of a state that a workgroup takes: 32, or 16 where 32 would make fewer than two workgroups a compute unit.  With 16 a chunk's matrices are read twice as often, with 32 its products
// take longer: one sequence of 32768 steps, 16 heads of 128 x 128: 16 columns 1061 us, 32 columns 1500; 5 prompts of 777, 6 heads of 96 x 80: 43 and 55; forward and backward of 8
// sequences of 2048, 16 heads of 128 x 128: 1246 and 1046, of 128 sequences of 25, 4 heads of 32 x 32 fp32: 92 and 82.
inline bool delta_narrow(int64_t B, int64_t heads, int64_t Dv) { return Dv <= 16 || B * heads * ((Dv + 31) / 32) < 2 * kFittedUnits; }

// A launch has a workgroup of up to 512 threads for every chunk and head, or for every 16 columns of a head: fewer than 2^32 threads.
inline bool delta_fits(int64_t T, int64_t B, int64_t heads, int64_t Dv) {
  const int64_t most = (1ll << 23) - 1;
  if (B * heads > most) return false;
  return delta_chunks(T) <= most / (B * heads) && (Dv + 15) / 16 <= most / (B * heads);
}

}  // namespace tac
