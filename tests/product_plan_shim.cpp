// The plan of a product of 8-bit matrices, for the tests of what it takes.
#include "tac_product_plan.h"

// out: tile (its place in kProductTiles), parts
extern "C" void product_plan_of(long long M, long long N, long long K, int bf16, int* out) {
  const tac::ProductPlan q = tac::choose_product_plan(M, N, K, bf16);
  out[0] = q.tile;
  out[1] = q.parts;
}

// rows, columns, workgroups that a compute unit takes; whether results of this type use it
extern "C" int product_tile_of(int tile, int bf16, int* out) {
  if (tile >= (int)(sizeof(tac::kProductTiles) / sizeof(tac::ProductTile))) return -1;
  const tac::ProductTile& t = tac::kProductTiles[tile];
  out[0] = t.rows;
  out[1] = t.cols;
  out[2] = t.shared;
  return t.block[bf16 != 0][0] > 0.0;
}

extern "C" int product_tile_lds(int rows, int cols, int waves, int stages) { return tac::tile_lds(rows, cols, waves, stages); }
