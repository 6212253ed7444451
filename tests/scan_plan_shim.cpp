// The waves of a workgroup of the gated recurrence, for the tests of what a launch holds.
#include "tac_scan_plan.h"

extern "C" int scan_waves_of(long long T, long long groups) { return tac::scan_waves(T, groups); }

extern "C" int rows_overlap_of(long long x, long long xt, long long xb, long long y, long long yt, long long yb, long long T, long long B, long long D, long long el) {
  return tac::rows_overlap({(const void*)x, xt, xb}, {(const void*)y, yt, yb}, T, B, D, el);
}
