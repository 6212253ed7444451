// Host rule of the conversions to 8 bits: which kernel, by what a launch can hold.
#pragma once
#include "tac_internal.h"

namespace tac {

constexpr int64_t kMostThreads = 1ll << 32;          // a launch has fewer threads along an axis
constexpr int64_t kMostTiles = kMostThreads / 256;   // tiles of 128 x 128 of a call

// Whether the kernel for rows alone is taken, which has 512 threads a tile; the one for rows and columns has 256, and gives the same codes of the rows.
inline bool rows_alone(bool columns, bool tiles, int64_t count) { return !columns && !tiles && 512 * count < kMostThreads; }

}  // namespace tac
