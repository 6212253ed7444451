// The host rules of the head norm and the gated delta rule, for the tests of what a launch holds.
#include "tac_delta_plan.h"

extern "C" {
int head_lanes_of(int D, int rotated) { return tac::head_lanes(D, rotated).lanes; }
int head_apart_of(int D, int rotated) { return tac::head_lanes(D, rotated).apart; }
int head_slices_of(long long rows, int heads, int lanes) { return tac::head_slices(rows, heads, lanes); }
long long head_groups_of(long long rows, int slices, int lanes, int backward) { return tac::head_groups(rows, slices, lanes, backward ? tac::kHeadBackwardGroups : tac::kHeadGroups); }
int delta_fits_of(long long T, long long B, long long heads, long long Dv) { return tac::delta_fits(T, B, heads, Dv); }
int delta_narrow_of(long long B, long long heads, long long Dv) { return tac::delta_narrow(B, heads, Dv); }
}
