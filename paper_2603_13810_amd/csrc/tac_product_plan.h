// Host rules of the products of 8-bit matrices: which tile, how many parts of the columns, and the LDS of a tile.
#pragma once
#include "tac_internal.h"

namespace tac {

constexpr int kBlock = TAC_SCALE_BLOCK;      // columns that share a scale

// LDS of product_tile_kernel: STAGES stages of the tile's rows, of which the last one's place also takes the results on their way out (32 rows of up to
// 256 bytes and 16 for each wave), then as many sets of scale bytes of four blocks.
constexpr int tile_scales_at(int TM, int TN, int waves, int STAGES) {
  const int stage = (TM + TN) * kBlock, out = waves * 32 * (256 + 16);
  return (STAGES - 1) * stage + (stage > out ? stage : out);
}
constexpr int tile_lds(int TM, int TN, int waves, int STAGES) { return tile_scales_at(TM, TN, waves, STAGES) + 256 * STAGES * waves; }

// The tile and the number of parts, by an estimate in microseconds: a launch, then for every round of workgroups a beginning and an end and the blocks
// of columns of an item.  Fitted to products on 256 compute units, with one to four workgroups on each; measured, M x N x K in us:
//   bfloat16 results         16384 x 8192 x 4096  4096^3  1024 x 4096 x 4096  2048^3  1500^3  512 x 4096 x 4096  256 x 4096 x 4096  16 x 8192 x 4096
//   256 x 256, 8 waves                       459      62                  45      26       -                 44                 42                41
//   128 x 128, 4 stages                      634      88                  23      14      15                 21                 19                19
//   128 x 128, 2 stages                      555      71                  28      13      14                 25                 19                22
//   64 x 64, 2 waves, 2 stages                 -     117                  31      17      13                 20                 12                17
//   64 x 64, 2 waves, 4 stages               983     126                  34      20      17                 18                 13                12
//   64 x 64, 4 waves, 4 stages                 -     152                  40      23      20                 21                 12                11
//   64 x 32, 2 waves, 8 stages                 -       -                   -       -       -                 -                  -                 9
//   float32 results          8192 x 4096 x 8192  2000 x 3000 x 1000  512 x 4096 x 4096  1500^3  3200 x 500 x 3136  128 x 3136 x 3200  500 x 700 x 900
//   256 x 256, 8 waves                      408                   -                  -       -                 62                 58               24
//   128 x 128, 2 stages                     474                  20                 33      17                 27                 25               12
//   128 x 64                                  -                  19                 24      16                 18                 16                8
//   64 x 64, 4 waves, 2 stages                -                  22                 26      15                 20                 12                6
// Large tiles read less per product, small ones give more workgroups and shorter blocks; stages hide memory where few workgroups do.  Parts cost
// their sums' way through memory: 128 x 3136 x 3200 float32 in one part 14.1 us, in two 13.1; 3200 x 500 x 3136 18 and 23.
// The last tile is for few rows, where the other matrix's bytes count: seven blocks on their way per compute unit. With it, weights from memory, bfloat16
// results: 16 x 8192 x 4096 14.9 -> 11.9 us, 64 x 8192 x 4096 16.8 -> 13.4, 100 x 4096 x 4096 12.9 -> 11.0.
struct ProductPlan {
  int tile, parts;
};
struct ProductTile {
  int rows, cols, shared;            // shared: workgroups that a compute unit takes
  double ends, block[2][4];          // block: of a workgroup that shares its unit with none, one, two, three others; float32 and bfloat16 results (0: not used)
};
constexpr ProductTile kProductTiles[] = {{256, 256, 1, 6.0, {{3.05}, {1.6}}},
                           {128, 128, 1, 3.0, {{}, {0.6}}},
                           {128, 128, 2, 3.0, {{1.0, 1.8}, {0.65, 1.02}}},
                           {128, 64, 2, 2.5, {{0.58, 0.88}, {}}},
                           {64, 64, 4, 2.0, {{}, {0.33, 0.47, 0.67, 0.85}}},
                           {64, 64, 2, 2.0, {{}, {0.3, 0.45}}},
                           {64, 64, 1, 2.0, {{}, {0.23}}},
                           {64, 64, 3, 2.0, {{0.45, 0.64, 0.9}, {}}},
                           {64, 32, 1, 2.0, {{}, {0.22}}}};

inline ProductPlan choose_product_plan(int64_t M, int64_t N, int64_t K, int bf) {
  const int64_t blocks = (K + kBlock - 1) / kBlock;
  ProductPlan best = {0, 1};
  double least = 1e300;
  for (int tile = 0; tile < (int)(sizeof(kProductTiles) / sizeof(ProductTile)); ++tile) {
    const ProductTile& q = kProductTiles[tile];
    const double* block = q.block[bf != 0];
    if (block[0] == 0.0) continue;
    const int64_t tiles = ((M + q.rows - 1) / q.rows) * ((N + q.cols - 1) / q.cols);
    for (int parts : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
      if (parts > 1 && (2 * parts > blocks || tiles * parts > 2 * kFittedUnits)) break;
      const int64_t items = tiles * parts, whole = kFittedUnits * q.shared, left = items % whole;
      const double each = (double)((blocks + parts - 1) / parts);
      double us = (double)(items / whole) * (q.ends + each * block[q.shared - 1]);
      if (left) us += q.ends + each * block[(left - 1) / kFittedUnits];
      if (parts > 1) us += 3.0 + (double)M * (double)N * (8.0 * parts + (bf ? 2.0 : 4.0)) / 4e6;
      if (us < least) {
        least = us;
        best = ProductPlan{tile, parts};
      }
    }
  }
  return best;
}

}  // namespace tac
