// Host rule of the gated recurrence: the waves of a workgroup.
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

}  // namespace tac
