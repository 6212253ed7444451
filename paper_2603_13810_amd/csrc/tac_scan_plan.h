// Host rules of the gated recurrence: the waves of a workgroup, and whether sequences lie on top of each other.
#pragma once
#include "tac_internal.h"

namespace tac {

constexpr int kScanWaves = 8;                        // most waves of a workgroup

// As many waves as there are chunks of steps, and fewer where `groups` workgroups of them would be 2^32 threads, which no launch holds (from 2^23 groups on; one
// wave always fits: B D < 2^31 and B < 2^16 are fewer than 2^26 groups of 64 channels).
inline int scan_waves(int64_t T, int64_t groups) {
  const int64_t chunks = (T + TAC_SCAN_CHUNK - 1) / TAC_SCAN_CHUNK, fit = ((1ll << 32) - 1) / (64 * groups);
  const int64_t waves = chunks < kScanWaves ? chunks : kScanWaves;
  return (int)(waves < fit ? waves : fit);
}

// T x B rows of D elements
struct Rows {
  const void* at;
  int64_t stride_t, stride_b;        // elements
};

// Whether two of them, of elements of `el` bytes, may share memory.  Slices of the same wider rows do not: the same strides, and next to each other within them.
inline bool rows_overlap(const Rows& x, const Rows& y, int64_t T, int64_t B, int64_t D, int64_t el) {
  auto span = [&](const Rows& r) { return ((T - 1) * r.stride_t + (B - 1) * r.stride_b + D) * el; };
  const int64_t from = (int64_t)(uintptr_t)x.at, to = (int64_t)(uintptr_t)y.at;
  if (from + span(x) <= to || to + span(y) <= from) return false;
  if ((T > 1 && x.stride_t != y.stride_t) || (B > 1 && x.stride_b != y.stride_b)) return true;
  const int64_t apart = from < to ? to - from : from - to;
  return apart < D * el || (T > 1 && apart + D * el > x.stride_t * el) || (B > 1 && apart + D * el > x.stride_b * el);
}

}  // namespace tac
