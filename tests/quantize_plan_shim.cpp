// The choice of the kernel that converts to 8 bits, for the tests of what a launch holds.
#include "tac_quantize_plan.h"

extern "C" int quantize_rows_alone(int columns, int tiles, long long count) { return tac::rows_alone(columns, tiles, count); }
extern "C" long long quantize_most_tiles() { return tac::kMostTiles; }
