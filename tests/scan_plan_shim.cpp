// The waves of a workgroup of the gated recurrence, for the tests of what a launch holds.
#include "tac_scan_plan.h"

extern "C" int scan_waves_of(long long T, long long groups) { return tac::scan_waves(T, groups); }
